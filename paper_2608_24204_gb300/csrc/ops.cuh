// Device helpers of the stand-alone operators: element types, the 8- and 4-bit cache formats.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "ops.h"

namespace wici {

// a tensor [tokens][heads][d] as a kernel sees it (strides in elements)
struct HeadsArg {
    void *data;
    int64_t ts, hs;
    template <typename T>
    __device__ __forceinline__ T *row(int64_t token, int head) const {
        return (T *)data + token * ts + (int64_t)head * hs;
    }
};
inline HeadsArg heads_arg(const wici_heads *t) {
    return t ? HeadsArg{t->data, t->token_stride, t->head_stride} : HeadsArg{nullptr, 0, 0};
}

struct CacheArg {
    uint8_t *data;
    int64_t page_stride;
    int n_pages, kv_heads;
};
inline CacheArg cache_arg(const wici_kv_cache *c) {
    return CacheArg{(uint8_t *)c->data, c->page_stride, c->n_pages, c->n_kv_heads};
}

__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ void from_f32(float f, __nv_bfloat16 &v) { v = __float2bfloat16_rn(f); }
__device__ __forceinline__ void from_f32(float f, __half &v) { v = __float2half_rn(f); }
__device__ __forceinline__ void from_f32(float f, float &v) { v = f; }

// the first n of 8 elements at p as fp32, one by one, zeros after them
template <typename T>
__device__ __forceinline__ void load8(const T *p, int n, float *v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? to_f32(p[j]) : 0.f;
}

// 8 elements in 16-byte stores (none where n is 0), or (WIDE false) the first n one by one
template <typename T, bool WIDE>
__device__ __forceinline__ void store8(T *p, int n, const float *v) {
    alignas(16) T e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) from_f32(v[j], e[j]);
    if (WIDE) {
        if (n > 0) {
            *(uint4 *)p = *(const uint4 *)e;
            if (sizeof(T) == 4) *((uint4 *)p + 1) = *((const uint4 *)e + 1);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = e[j];
}

// ---------------------------------------------------------- 8-bit cache formats
// the smallest NaN-or-infinity pattern of |x|: larger patterns are larger values or NaNs
constexpr uint32_t kInfBits = 0x7F800000u;

// The codes of 16 values of a head whose largest magnitude is `top` (NaN where one is); the scale is returned.
// Quotients of bf16 values often lie on a code's border, so a product with one reciprocal r a head has to be mended by
// its remainder (an operation or two an element, against ten of a division).  A scale below the normal range, whose
// reciprocal might overflow, is 0: such a head is below 2^-117.
//   int8: x r, off by less than 2^-16, goes to an integer n; e = x - n scale is exact near half a scale and beyond (a
//   multiple of half the scale's last place there), and moves n where it is more than half a scale, or just that and n odd.
//   So a code is x / scale itself rounded to nearest even, not a quotient that was rounded before.  Four elements at a
//   time are looked at whether one has to move: 16384 tokens, 32 q heads rotated, 8 k and v heads in bf16, and read back
//   89.6 us (89.5 where the fp32 quotient is rounded; 94.0 with each element's move computed), in fp32 133.8 (133.3; 135.3).
//   e4m3: x r + (x - x r scale) r is the fp32 quotient, right to its last bit, and that is rounded.
template <int FMT>
__device__ __forceinline__ float quantise16(const float *x, float top, uint32_t *code) {
#pragma unroll
    for (int j = 0; j < 4; ++j) code[j] = 0;
    if (!(top < __uint_as_float(kInfBits))) return __uint_as_float(0x7FC00000u);   // an infinity or NaN among them
    const float scale = top / (FMT == WICI_KV_INT8 ? 127.f : 448.f);
    if (scale < 0x1p-126f) return 0.f;
    const float r = 1.f / scale;
    if (FMT == WICI_KV_INT8) {
        constexpr float kInteger = 12582912.f;       // 1.5 * 2^23: plus n, it has n in its low byte
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t b[4];
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y = fmaf(x[4 * j + i], r, kInteger);
                most = fmaxf(most, fabsf(fmaf(kInteger - y, scale, x[4 * j + i])));
                b[i] = __float_as_uint(y);
            }
            if (most + most >= scale) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = fmaf(kInteger - __uint_as_float(b[i]), scale, x[4 * j + i]);
                    // positive floats compare as their bits do
                    if (__float_as_uint(fabsf(e + e)) + (b[i] & 1) > __float_as_uint(scale)) b[i] += e < 0.f ? -1 : 1;
                }
            }
            code[j] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = x[4 * j + i] * r;
                y[i] = fmaf(fmaf(-y[i], scale, x[4 * j + i]), r, y[i]);
            }
            code[j] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3) |
                      (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[2], y[3]), __NV_SATFINITE, __NV_E4M3) << 16;
        }
    }
    return scale;
}

// The four codes of w as two fp16 pairs, exactly.  An int8 code c is the fp16 number 1024 + (c + 128) less 1152.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if (FMT == WICI_KV_INT8) {
        const uint32_t x = w ^ 0x80808080u;
        const uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
        const __half2 off = __half2half2(__ushort_as_half((unsigned short)0x6480));   // 1152
        const __half2 p = __hsub2(*(const __half2 *)&a, off), q = __hsub2(*(const __half2 *)&b, off);
        lo = *(const uint32_t *)&p;
        hi = *(const uint32_t *)&q;
    } else {
        const __half2 p = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xFFFF), __NV_E4M3));
        const __half2 q = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3));
        lo = *(const uint32_t *)&p;
        hi = *(const uint32_t *)&q;
    }
}

// ------------------------------------------------------------ 4-bit cache format
// e2m1 codes c of 16 elements share an e4m3 scale b, and a head's elements an fp32 scale s: c b s.  c b has at most 6
// significant bits between 2^-10 and 2688: fp16 holds it exactly.
//
// Which code a value gets is decided on the real numbers, not on rounded quotients, for bf16 values often lie half way
// between two codes: x goes to the upper of two neighbours where x > m b s with m their middle, and fmaf(-m b, s, x) has
// that difference's sign, for m b is exact (7 bits).  Nearly always a quotient within 2^-19 tells without it.
constexpr float kE2m1Top = 2688.f;               // 6 * 448
constexpr float kE2m1Least = 0x1p-100f;          // smaller scales are 0: with block scales, reciprocals and products stay normal
constexpr float kNearLo = 1.f - 0x1p-19f, kNearHi = 1.f + 0x1p-19f;

// the e4m3 nearest to most / (6 scale), the even one of two that are as near; per6 is about 1 / (6 scale)
__device__ __forceinline__ uint32_t block_scale(float most, float scale, float per6) {
    const float y = most * per6;
    const uint32_t w = __nv_cvt_float2_to_fp8x2(make_float2(y * kNearLo, y * kNearHi), __NV_SATFINITE, __NV_E4M3);
    const uint32_t lo = w & 0xFF, hi = w >> 8;
    if (lo == hi) return lo;
    const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3)));
    const float over = fmaf(-3.f * (v.x + v.y), scale, most);
    return over > 0.f || (over == 0.f && (hi & 1) == 0) ? hi : lo;
}
__device__ __forceinline__ float e4m3_value(uint32_t code) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}
// about 1 / x, of a normal x up to 2^126: within 2^-22 of it
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 8 values times r as the nearest codes, the first in the lowest bits
__device__ __forceinline__ uint32_t encode_e2m1(const float *x, float r) {
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w)
        : "f"(x[0] * r), "f"(x[1] * r), "f"(x[2] * r), "f"(x[3] * r), "f"(x[4] * r), "f"(x[5] * r), "f"(x[6] * r), "f"(x[7] * r));
    return w;
}
// Quotients of values of 11 bits at most (16-bit types) with the row's largest such value need no second look.  x / (b s)
// with s = top / 2688 unrounded is 21 X 2^k / (T B), with integers X, T < 2^11 and B < 2^4: it is a middle m / 2^j, m < 2^3,
// or off by 2^-18 of it and more (2^-16 for a block scale's).  s being off by 2^-24, a quotient within 2^-19 of a middle is
// that middle moved by s's own rounding, to the same side for a whole row: 2^-20 that way decides it, beside errors of 2^-21.
// `left`: what top has over 2688 s; 0, where such quotients are middles exactly, is not for this.
__device__ __forceinline__ float nudge_of(float left) { return left > 0.f ? 1.f + 0x1p-20f : 1.f - 0x1p-20f; }
// the codes of 8 values under the block scale b (its value) and the head's scale, the first in the lowest bits
__device__ __forceinline__ uint32_t quantise_e2m1(const float *x, float b, float scale) {
    const float r = b > 0.f ? reciprocal(b * scale) : 0.f;
    uint32_t lo = encode_e2m1(x, r * kNearLo);
    const uint32_t hi = encode_e2m1(x, r * kNearHi);
    // values of few bits are often on a middle: one lane or two of most warps have one, so it is one place at a time (all 8
    // in turn: 34 in place of 32 us for 16384 tokens of 16 rows in bf16, before 16-bit values had a way of their own)
    for (uint32_t differ = lo ^ hi; differ;) {
        const int at = (31 - __clz(differ)) & ~3, j = at >> 2;
        differ &= (1u << at) - 1;
        const float x0 = j & 1 ? x[1] : x[0], x2 = j & 1 ? x[3] : x[2], x4 = j & 1 ? x[5] : x[4], x6 = j & 1 ? x[7] : x[6];
        const float x04 = j & 4 ? x4 : x0, x26 = j & 4 ? x6 : x2, xj = j & 2 ? x26 : x04;
        const uint32_t c = lo >> at & 7;         // the lower neighbour
        const float middle = c < 4 ? 0.25f + 0.5f * (float)c : c == 4 ? 2.5f : c == 5 ? 3.5f : 5.f;
        const float over = fmaf(-middle * b, scale, fabsf(xj));
        if (over > 0.f || (over == 0.f && (c & 1))) lo += 1u << at;
    }
    return lo;
}
// 8 codes as fp16 pairs, exactly
__device__ __forceinline__ void decode_e2m1(uint32_t w, uint32_t *h) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}

}  // namespace wici
