// Attention of one new token per sequence over a paged key-value cache (include/wici_ops.h).
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "kernels.h"
#include "ops.cuh"

using namespace wici;

namespace {

int fail(int code, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_thread_error(buf);
    return code;
}

constexpr int kAttnWarps = 4;

struct AttnArg {
    HeadsArg q, out;
    CacheArg cache;
    const int32_t *pages, *lengths;
    float *lse;
    int32_t *status;
    int q_heads, group, max_pages, window;
    int q_dtype, out_dtype;
    float scale;
};

__device__ __forceinline__ float load_any(const HeadsArg &t, int dtype, int64_t token, int head, int i) {
    switch (dtype) {
        case WICI_BF16: return to_f32(t.row<__nv_bfloat16>(token, head)[i]);
        case WICI_F16: return to_f32(t.row<__half>(token, head)[i]);
        default: return t.row<float>(token, head)[i];
    }
}

__device__ __forceinline__ void store_any(const HeadsArg &t, int dtype, int64_t token, int head, int i, float v) {
    switch (dtype) {
        case WICI_BF16: from_f32(v, t.row<__nv_bfloat16>(token, head)[i]); break;
        case WICI_F16: from_f32(v, t.row<__half>(token, head)[i]); break;
        default: t.row<float>(token, head)[i] = v; break;
    }
}

// One block per sequence and query head; a warp takes every fourth key and keeps the running
// maximum and sum of the softmax (s - max in fp32), a lane D / 32 adjacent elements of the head.
template <int FMT, int D>
__global__ void __launch_bounds__(32 * kAttnWarps) attention_kernel(const __grid_constant__ AttnArg a) {
    constexpr int E = D / 32;
    __shared__ float sm[kAttnWarps], sl[kAttnWarps], so[kAttnWarps][D];
    griddep_wait();
    const int h = blockIdx.x, b = blockIdx.y, kvh = h / a.group;
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const int n = a.lengths[b];
    const int lo = a.window && n > a.window ? n - a.window : 0;
    bool bad = n > a.max_pages * (int64_t)kKvPage;
    int bits = bad ? WICI_BAD_LENGTH : 0;
    float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) q[e] = load_any(a.q, a.q_dtype, b, h, lane * E + e) * a.scale;
    for (int t = lo + warp; t < n && !bad; t += kAttnWarps) {
        const int page = a.pages[(int64_t)b * a.max_pages + t / kKvPage], place = t % kKvPage;
        if (page < 0 || page >= a.cache.n_pages) {
            bad = true;
            bits |= WICI_BAD_PAGE;
            break;
        }
        constexpr int64_t kBlock = FMT == WICI_KV_BF16 ? kKvPage * D * 2 : kKvPage * (D + 4);
        const uint8_t *kb = a.cache.data + page * a.cache.page_stride + kvh * kBlock;
        const uint8_t *vb = kb + a.cache.kv_heads * kBlock;
        float k[E], v[E];
        if (FMT == WICI_KV_BF16) {
            for (int e = 0; e < E; ++e) {
                k[e] = to_f32(((const __nv_bfloat16 *)kb)[place * D + lane * E + e]);
                v[e] = to_f32(((const __nv_bfloat16 *)vb)[place * D + lane * E + e]);
            }
        } else {
            const float ks = ((const float *)(kb + kKvPage * D))[place], vs = ((const float *)(vb + kKvPage * D))[place];
            for (int e = 0; e < E; e += 2) {
                const float2 k2 = __half22float2(decode2<FMT>(*(const uint16_t *)(kb + place * D + lane * E + e)));
                const float2 v2 = __half22float2(decode2<FMT>(*(const uint16_t *)(vb + place * D + lane * E + e)));
                k[e] = k2.x * ks;
                k[e + 1] = k2.y * ks;
                v[e] = v2.x * vs;
                v[e + 1] = v2.y * vs;
            }
        }
        float s = 0.f;
        for (int e = 0; e < E; ++e) s += q[e] * k[e];
        s = warp_sum(s);
        const float m2 = fmaxf(m, s), c = m2 == -INFINITY ? 1.f : expf(m - m2), p = s == -INFINITY ? 0.f : expf(s - m2);
        l = l * c + p;
        for (int e = 0; e < E; ++e) o[e] = o[e] * c + p * v[e];
        m = m2;
    }
    if (lane == 0) {
        sm[warp] = m;
        sl[warp] = l;
        if (bits && a.status) atomicOr(a.status, bits);
    }
    for (int e = 0; e < E; ++e) so[warp][lane * E + e] = o[e];
    bad = __syncthreads_or(bad);
    if (threadIdx.x < D) {
        float top = -INFINITY, sum = 0.f, acc = 0.f;
        for (int w = 0; w < kAttnWarps; ++w) top = fmaxf(top, sm[w]);
        for (int w = 0; w < kAttnWarps; ++w) {
            const float c = sm[w] == -INFINITY ? 0.f : expf(sm[w] - top);
            sum += sl[w] * c;
            acc += so[w][threadIdx.x] * c;
        }
        const float nan = __uint_as_float(0x7FC00000u);
        store_any(a.out, a.out_dtype, b, h, threadIdx.x, bad ? nan : sum > 0.f ? acc / sum : acc);
        if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)b * a.q_heads + h] = bad ? nan : top + logf(sum);
    }
}

template <int FMT>
cudaError_t launch(int d, const AttnArg &a, int batch, cudaStream_t st) {
    const dim3 grid(a.q_heads, batch);
    return d == 64 ? launch_kernel(attention_kernel<FMT, 64>, grid, 32 * kAttnWarps, 0, st, 1, true, a)
                   : launch_kernel(attention_kernel<FMT, 128>, grid, 32 * kAttnWarps, 0, st, 1, true, a);
}

const char *check_query_heads(const wici_kv_cache *c, int n_q_heads) {
    return n_q_heads < 1 || n_q_heads > kMaxHeads || n_q_heads % c->n_kv_heads
               ? "query heads must be a multiple of the cache's heads"
               : nullptr;
}

}  // namespace

extern "C" {

int wici_paged_attention_workspace_bytes(const wici_kv_cache *cache, int32_t n_q_heads, int32_t batch, size_t *bytes) {
    if (const char *m = check_cache(cache)) return fail(WICI_E_ARG, "attention: %s", m);
    if (const char *m = check_query_heads(cache, n_q_heads)) return fail(WICI_E_ARG, "attention: %s", m);
    if (batch < 0 || batch > 65535) return fail(WICI_E_ARG, "attention: batch must be in [0, 65535]");
    if (!bytes) return fail(WICI_E_ARG, "attention: null output");
    *bytes = 256;
    return WICI_OK;
}

int wici_paged_attention(void *cuda_stream, const wici_kv_cache *cache, const wici_attn_shape *shape,
                         const int32_t *pages, const int32_t *lengths, const wici_heads *q, const wici_heads *out,
                         float *lse, void *workspace, int32_t *status) {
    if (const char *m = check_cache(cache)) return fail(WICI_E_ARG, "attention: %s", m);
    if (!shape) return fail(WICI_E_ARG, "attention: null shape");
    if (shape->batch < 0 || shape->batch > 65535) return fail(WICI_E_ARG, "attention: batch must be in [0, 65535]");
    if (shape->max_pages < 1 || shape->max_pages > kMaxPages)
        return fail(WICI_E_ARG, "attention: max_pages must be in [1, 2^27)");
    if (shape->window < 0) return fail(WICI_E_ARG, "attention: window must be >= 0");
    if (!isfinite(shape->scale)) return fail(WICI_E_ARG, "attention: scale must be finite");
    if (const char *m = check_heads(q, shape->batch, cache->head_dim, false)) return fail(WICI_E_ARG, "attention q: %s", m);
    if (const char *m = check_heads(out, shape->batch, cache->head_dim, true))
        return fail(WICI_E_ARG, "attention out: %s", m);
    if (q->heads != out->heads) return fail(WICI_E_ARG, "attention: q and out differ in heads");
    if (const char *m = check_query_heads(cache, q->heads)) return fail(WICI_E_ARG, "attention: %s", m);
    if (shape->batch == 0) return WICI_OK;
    if (!pages || !lengths || !workspace || ((uintptr_t)workspace & 15))
        return fail(WICI_E_ARG, "attention: null pages or lengths, or workspace null or not 16-byte aligned");
    AttnArg a = {};
    a.q = heads_arg(q);
    a.out = heads_arg(out);
    a.cache = cache_arg(cache);
    a.pages = pages;
    a.lengths = lengths;
    a.lse = lse;
    a.status = status;
    a.q_heads = q->heads;
    a.group = q->heads / cache->n_kv_heads;
    a.max_pages = shape->max_pages;
    a.window = shape->window;
    a.q_dtype = q->dtype;
    a.out_dtype = out->dtype;
    a.scale = shape->scale;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    switch (cache->format) {
        case WICI_KV_BF16: e = launch<WICI_KV_BF16>(cache->head_dim, a, shape->batch, st); break;
        case WICI_KV_INT8: e = launch<WICI_KV_INT8>(cache->head_dim, a, shape->batch, st); break;
        default: e = launch<WICI_KV_E4M3>(cache->head_dim, a, shape->batch, st); break;
    }
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "attention: %s", cudaGetErrorString(e));
}

}  // extern "C"
