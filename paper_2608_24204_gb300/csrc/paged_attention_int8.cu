// Paged attention over an int8 cache.
#include "paged_attention.cuh"

namespace wici {

cudaError_t launch_attention_int8(int d, const AttnArg &a, bool stack, int grid, cudaStream_t st) {
    if (d == 64)
        return stack ? launch_attention<WICI_KV_INT8, 64, true, false>(a, grid, st)
                     : launch_attention<WICI_KV_INT8, 64, false, false>(a, grid, st);
    return stack ? launch_attention<WICI_KV_INT8, 128, true, false>(a, grid, st)
                 : launch_attention<WICI_KV_INT8, 128, false, false>(a, grid, st);
}

cudaError_t setup_attention_int8() {
    cudaError_t e = limit_attention<WICI_KV_INT8, 64, true, false>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_INT8, 64, false, false>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_INT8, 128, true, false>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_INT8, 128, false, false>();
    return e;
}

}  // namespace wici
