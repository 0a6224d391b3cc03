// Attention of one new token per sequence over a paged key-value cache (include/wici_ops.h):
// argument checks and launches.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "device_table.h"
#include "kernels.h"
#include "paged_attention.cuh"

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

DeviceTable<int> g_sms;

// the current device's SMs, with the kernels' shared-memory limits set there
int device_sms(int *n) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = g_sms.get(dev, n, [dev](int *d) {
        cudaError_t e1 = setup_attention_bf16();
        if (e1 == cudaSuccess) e1 = setup_attention_int8();
        if (e1 == cudaSuccess) e1 = setup_attention_e4m3();
        if (e1 != cudaSuccess) return e1;
        return cudaDeviceGetAttribute(d, cudaDevAttrMultiProcessorCount, dev);
    });
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "attention setup: %s", cudaGetErrorString(e));
}

constexpr int kTicketBytes = WICI_ATTN_ZEROED;   // arrivals of every block: zero before the first launch, and after each
constexpr int kBlocksPerSm = AttnShape<WICI_KV_BF16, 128, true>::kBlocks;   // of every kernel
// SMs that a launch uses: tickets are for so many blocks
int used_sms(int sms) {
    const int most = kTicketBytes / (int)sizeof(int) / kBlocksPerSm;
    return sms < most ? sms : most;
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
    int sms = 152;   // without a device: a GB300's
    int dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess) {
        if (int rc = device_sms(&sms)) return rc;
    } else {
        cudaGetLastError();
    }
    *bytes = kTicketBytes + (size_t)used_sms(sms) * kBlocksPerSm * 2 * attn_piece_floats(cache->head_dim) * sizeof(float);
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
    if ((int64_t)(shape->max_pages + 2) * q->heads >= (int64_t)1 << 31)
        return fail(WICI_E_ARG, "attention: (max_pages + 2) * heads must be below 2^31");
    if (shape->batch == 0) return WICI_OK;
    if (!pages || !lengths || !workspace || ((uintptr_t)workspace & 15))
        return fail(WICI_E_ARG, "attention: null pages or lengths, or workspace null or not 16-byte aligned");
    if (!words(pages) || !words(lengths) || !words(lse) || !words(status))
        return fail(WICI_E_ARG, "attention: pages, lengths, lse or status unaligned");
    int sms = 0;
    if (int rc = device_sms(&sms)) return rc;
    AttnArg a = {};
    a.q = heads_arg(q);
    a.out = heads_arg(out);
    a.cache = cache_arg(cache);
    a.status = status;
    a.tickets = (int *)workspace;
    a.pieces = (float *)((uint8_t *)workspace + kTicketBytes);
    a.q_heads = q->heads;
    a.group = q->heads / cache->n_kv_heads;
    // more terms where fp32 comes in or, over a bf16 cache, goes out or q is not bf16
    const bool exact = cache->format == WICI_KV_BF16 ? q->dtype != WICI_BF16 || out->dtype == WICI_F32 : q->dtype == WICI_F32;
    const AttnKind kind = attn_kind(a.group, exact);
    a.tiles = kind == ATTN_PLAIN ? (a.group + 15) / 16 : (a.group + 7) / 8;
    a.max_pages = shape->max_pages;
    a.window = shape->window;
    a.q_dtype = q->dtype;
    a.out_dtype = out->dtype;
    a.q_wide = wide_heads(q);
    a.out_wide = wide_heads(out);
    a.scale = shape->scale;
    // the weight of a launch's segments adds up in 31 bits
    const int64_t each = ((int64_t)shape->max_pages + kAttnSegment) * cache->n_kv_heads * a.tiles, room = INT32_MAX / each;
    const int fit = kind == ATTN_PLAIN ? AttnShape<WICI_KV_BF16, 128, false>::kMaxBatch : AttnShape<WICI_KV_BF16, 128, true>::kMaxBatch;
    const int most = room < 1 ? 1 : room < fit ? (int)room : fit;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    for (int b = 0; b < shape->batch && e == cudaSuccess; b += most) {
        a.batch = shape->batch - b < most ? shape->batch - b : most;
        a.pages = pages + (int64_t)b * shape->max_pages;
        a.lengths = lengths + b;
        a.lse = lse ? lse + (int64_t)b * q->heads : nullptr;
        a.q.data = (uint8_t *)q->data + (int64_t)b * q->token_stride * dtype_bytes(q->dtype);
        a.out.data = (uint8_t *)out->data + (int64_t)b * out->token_stride * dtype_bytes(out->dtype);
        switch (cache->format) {
            case WICI_KV_BF16: e = launch_attention_bf16(cache->head_dim, a, kind, used_sms(sms), st); break;
            case WICI_KV_INT8: e = launch_attention_int8(cache->head_dim, a, kind, used_sms(sms), st); break;
            default: e = launch_attention_e4m3(cache->head_dim, a, kind, used_sms(sms), st); break;
        }
    }
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "attention: %s", cudaGetErrorString(e));
}

}  // extern "C"
