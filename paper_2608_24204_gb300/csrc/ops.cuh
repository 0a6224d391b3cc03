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

// 8 elements at p as fp32: 16-byte loads, or (WIDE false) the first n one by one, zeros after them
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T *p, int n, float *v) {
    if (WIDE) {
        if (n > 0) {
            alignas(16) T e[8];
            if (sizeof(T) == 4) {
                *(uint4 *)e = *(const uint4 *)p;
                *((uint4 *)e + 1) = *((const uint4 *)p + 1);
            } else {
                *(uint4 *)e = *(const uint4 *)p;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
            return;
        }
        n = 0;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? to_f32(p[j]) : 0.f;
}

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
template <int FMT>
__device__ __forceinline__ float largest_code() {
    return FMT == WICI_KV_INT8 ? 127.f : 448.f;
}

// four codes of x / scale, rounded to nearest even (scale > 0)
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float *x, float scale) {
    if (FMT == WICI_KV_INT8) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // a scale below the normal range is rounded coarsely: the quotient may pass 127
            const int c = __float2int_rn(fminf(fmaxf(x[j] / scale, -127.f), 127.f));
            w |= (uint32_t)(c & 255) << (8 * j);
        }
        return w;
    }
    const __nv_fp8x2_storage_t lo =
        __nv_cvt_float2_to_fp8x2(make_float2(x[0] / scale, x[1] / scale), __NV_SATFINITE, __NV_E4M3);
    const __nv_fp8x2_storage_t hi =
        __nv_cvt_float2_to_fp8x2(make_float2(x[2] / scale, x[3] / scale), __NV_SATFINITE, __NV_E4M3);
    return (uint32_t)lo | (uint32_t)hi << 16;
}

// two codes (the low half of w) as fp16, exactly
template <int FMT>
__device__ __forceinline__ __half2 decode2(uint32_t w) {
    if (FMT == WICI_KV_INT8)
        return __halves2half2(__int2half_rn((int8_t)(w & 255)), __int2half_rn((int8_t)((w >> 8) & 255)));
    return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xFFFF), __NV_E4M3));
}

// the smallest NaN-or-infinity pattern of |x|: larger patterns are larger values or NaNs
constexpr uint32_t kInfBits = 0x7F800000u;

}  // namespace wici
