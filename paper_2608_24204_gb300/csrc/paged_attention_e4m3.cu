// Paged attention over an e4m3 cache.
#include "paged_attention.cuh"

namespace wici {

cudaError_t launch_attention_e4m3(int d, const AttnArg &a, bool stack, int grid, cudaStream_t st) {
    if (d == 64)
        return stack ? launch_attention<WICI_KV_E4M3, 64, true, false>(a, grid, st)
                     : launch_attention<WICI_KV_E4M3, 64, false, false>(a, grid, st);
    return stack ? launch_attention<WICI_KV_E4M3, 128, true, false>(a, grid, st)
                 : launch_attention<WICI_KV_E4M3, 128, false, false>(a, grid, st);
}

cudaError_t setup_attention_e4m3() {
    cudaError_t e = limit_attention<WICI_KV_E4M3, 64, true, false>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_E4M3, 64, false, false>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_E4M3, 128, true, false>();
    if (e == cudaSuccess) e = limit_attention<WICI_KV_E4M3, 128, false, false>();
    return e;
}

}  // namespace wici
