// Paged attention over an int8 cache.
#include "paged_attention.cuh"

namespace wici {

template <int D>
static cudaError_t launch_d(const AttnArg &a, AttnKind kind, int sms, cudaStream_t st) {
    switch (kind) {
        case ATTN_STACK: return launch_attention<WICI_KV_INT8, D, true, false>(a, sms, st);
        case ATTN_STACK_EXACT: return launch_attention<WICI_KV_INT8, D, true, true>(a, sms, st);
        default: return launch_attention<WICI_KV_INT8, D, false, false>(a, sms, st);
    }
}

cudaError_t launch_attention_int8(int d, const AttnArg &a, AttnKind kind, int sms, cudaStream_t st) {
    return d == 64 ? launch_d<64>(a, kind, sms, st) : launch_d<128>(a, kind, sms, st);
}

template <int D>
static cudaError_t setup_d() {
    cudaError_t e = limit_attention<WICI_KV_INT8, D, true, false>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_INT8, D, true, true>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_INT8, D, false, false>();
    return e;
}

cudaError_t setup_attention_int8() {
    const cudaError_t e = setup_d<64>();
    return e == cudaSuccess ? setup_d<128>() : e;
}

}  // namespace wici
