// Device helpers of the stand-alone operators: element types, the 8-bit cache formats.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
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


}  // namespace wici
