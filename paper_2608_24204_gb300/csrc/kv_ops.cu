// Rotary positions, and writing and reading a paged key-value cache (include/wici_ops.h).
//
// The three are row-wise: a row is one head of one token, cut into chunks of 16 elements, one
// lane each.  All are bound by HBM (each element is read and written once; a rotation is 6
// operations a pair, a quantisation one division an element), and by launch latency when the
// call is a step of few tokens.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "device_table.h"
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

constexpr int kRowThreads = 256;
constexpr int kBlockTokens = 16;      // tokens of a block at most: their angles are in shared memory
constexpr int kRopeOnly = -1;         // FMT of a launch without a cache

struct RopeArg {
    uint64_t turns[128];
    float gain, sign;
    int head_dim, rot, interleaved;
};

struct RowsArg {
    RopeArg rope;
    HeadsArg q, q_out, k, v;
    CacheArg cache;
    const int32_t *positions, *slots;
    int32_t *status;
    int64_t tokens;
    int q_heads, heads;               // rows of a token: q heads, then (with a cache) k heads and v heads
    int block_tokens, block_heads;
    int chunks, rot_chunks;           // lanes of a row, those of them that hold rotated pairs
    bool rotate_k;
};

// cos and sin of the angle that is `phase` / 2^64 of a turn.  The quadrant is taken off in
// integers, so the fp32 argument is at most an eighth of a turn and exact to 2^-24 of itself:
// the angle is as good at position 10^6 as at position 1.
__device__ __forceinline__ float2 turn_of(uint64_t phase) {
    const int32_t t = (int32_t)(phase >> 32);                    // 2^-32 turns, wrapped to [-1/2, 1/2)
    const int quad = (int)(((uint32_t)t + 0x20000000u) >> 30);   // nearest quarter turn
    const int32_t rest = (int32_t)((uint32_t)t - ((uint32_t)quad << 30));
    float s, c;
    sincospif((float)rest * 0x1p-31f, &s, &c);
    if (quad & 1) {
        const float u = c;
        c = -s;
        s = u;
    }
    if (quad & 2) {
        c = -c;
        s = -s;
    }
    return make_float2(c, s);
}

// One launch rotates q rows (FMT = kRopeOnly: all rows) and writes k and v rows into the cache.
// A block takes block_tokens tokens (or block_heads heads of one): it computes their cosines
// and sines once, one pair a thread, then every row reads them from shared memory.
template <typename T, int FMT, bool WIDE>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const __grid_constant__ RowsArg a) {
    extern __shared__ float4 cs[];    // [token][4][rot_chunks]: (cos, sin) of pairs 8 chunk + 2 j, + 2 j + 1
    griddep_wait();
    const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens;
    const int nt = (int)(a.tokens - t0 < a.block_tokens ? a.tokens - t0 : a.block_tokens);
    const int h0 = blockIdx.y * a.block_heads;
    const int nh = a.heads - h0 < a.block_heads ? a.heads - h0 : a.block_heads;
    const int half = a.rope.rot / 2;
    const int tid = threadIdx.y * blockDim.x + threadIdx.x, nthreads = blockDim.x * blockDim.y;
    if (a.positions) {
        const int pairs = 8 * a.rot_chunks;
        for (int i = tid; i < nt * pairs; i += nthreads) {
            const int t = i / pairs, p = i - t * pairs;
            float2 w = make_float2(1.f, 0.f);
            if (p < half) {
                w = turn_of((uint64_t)(int64_t)a.positions[t0 + t] * a.rope.turns[p]);
                w.x *= a.rope.gain;
                w.y *= a.rope.gain * a.rope.sign;
            }
            ((float2 *)cs)[(((t * 4 + (p & 7) / 2) * a.rot_chunks + p / 8) << 1) + (p & 1)] = w;
        }
        __syncthreads();
    }
    const int c = threadIdx.x;
    const int rows = nt * nh;
    for (int base = 0; base < rows; base += blockDim.y) {   // every lane of a warp stays: rows are reduced by shuffles
        const int idx = base + threadIdx.y;
        const bool live = idx < rows;
        const int tl = live ? idx / nh : 0;
        const int64_t t = t0 + tl;
        int h = h0 + (live ? idx - tl * nh : 0);
        const bool is_q = FMT == kRopeOnly || h < a.q_heads;
        const bool is_v = !is_q && h >= a.q_heads + a.cache.kv_heads;
        if (!is_q) h -= a.q_heads + (is_v ? a.cache.kv_heads : 0);
        const bool rotate = is_q || (!is_v && a.rotate_k);
        // the chunk's two groups of 8: where they start, how many they hold
        int o0, o1, n0, n1;
        if (!rotate) {
            o0 = 16 * c;
            o1 = o0 + 8;
            n0 = n1 = 8;              // head_dim is 64 or 128 here
        } else if (c < a.rot_chunks) {
            const int n = half - 8 * c < 8 ? half - 8 * c : 8;
            if (a.rope.interleaved) {
                o0 = 16 * c;
                o1 = o0 + 8;
                n0 = 2 * n < 8 ? 2 * n : 8;
                n1 = 2 * n - n0;
            } else {
                o0 = 8 * c;
                o1 = half + 8 * c;
                n0 = n1 = n;
            }
        } else {
            o0 = a.rope.rot + 16 * (c - a.rot_chunks);
            o1 = o0 + 8;
            const int n = a.rope.head_dim - o0 < 16 ? a.rope.head_dim - o0 : 16;
            n0 = n < 8 ? n : 8;
            n1 = n - n0;
        }
        float x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = 0.f;
        if (live) {
            const T *src = (is_q ? a.q : is_v ? a.v : a.k).template row<T>(t, h);
            load8<T, WIDE>(src + o0, n0, x);
            load8<T, WIDE>(src + o1, n1, x + 8);
        }
        if (rotate && c < a.rot_chunks) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 w = cs[(tl * 4 + j) * a.rot_chunks + c];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int p = 2 * j + u;
                    const float co = u ? w.z : w.x, si = u ? w.w : w.y;
                    // both layouts with static register names
                    const float xa = a.rope.interleaved ? x[2 * p] : x[p];
                    const float xb = a.rope.interleaved ? x[2 * p + 1] : x[p + 8];
                    const float ya = xa * co - xb * si, yb = xa * si + xb * co;
                    if (a.rope.interleaved) {
                        x[2 * p] = ya;
                        x[2 * p + 1] = yb;
                    } else {
                        x[p] = ya;
                        x[p + 8] = yb;
                    }
                }
            }
        }
        if (is_q) {
            if (live) {
                T *dst = a.q_out.template row<T>(t, h);
                store8<T, WIDE>(dst + o0, n0, x);
                store8<T, WIDE>(dst + o1, n1, x + 8);
            }
        }
        if (FMT != kRopeOnly) {
            int slot = -1;
            if (live && !is_q) {
                slot = a.slots[t];
                if (slot >= a.cache.n_pages * kKvPage) {
                    if (a.status) atomicOr(a.status, WICI_BAD_SLOT);
                    slot = -1;
                }
            }
            const int d = 16 * a.chunks;
            uint8_t *block = a.cache.data + (int64_t)(slot / kKvPage) * a.cache.page_stride +
                             (int64_t)(is_v ? a.cache.kv_heads + h : h) *
                                 (FMT == WICI_KV_BF16 ? kKvPage * d * 2 : kKvPage * (d + 4));
            const int place = slot & (kKvPage - 1);
            if (FMT == WICI_KV_BF16) {
                if (slot >= 0) {
                    __nv_bfloat16 *dst = (__nv_bfloat16 *)block + place * d;
                    store8<__nv_bfloat16, true>(dst + o0, 8, x);
                    store8<__nv_bfloat16, true>(dst + o1, 8, x + 8);
                }
            } else {
                // the row's largest magnitude, as a bit pattern: infinities and NaNs are the largest
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
                for (int o = a.chunks / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                if (slot >= 0) {
                    float scale = __uint_as_float(top) / largest_code<FMT>();
                    uint32_t code[4] = {0, 0, 0, 0};
                    if (top >= kInfBits) {
                        scale = __uint_as_float(0x7FC00000u);
                    } else if (scale > 0.f) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) code[j] = encode4<FMT>(x + 4 * j, scale);
                    }
                    uint8_t *dst = block + place * d;
                    *(uint2 *)(dst + o0) = make_uint2(code[0], code[1]);
                    *(uint2 *)(dst + o1) = make_uint2(code[2], code[3]);
                    if (c == 0) ((float *)(block + kKvPage * d))[place] = scale;
                }
            }
        }
    }
}

struct ReadArg {
    HeadsArg k, v;
    CacheArg cache;
    const int32_t *slots;
    int32_t *status;
    int64_t tokens;
    int heads;                        // rows of a token: those of k, then those of v
    int block_tokens, block_heads;
    bool has_k;
};

// A row of the cache to a row of k or v.
template <typename T, int FMT, int D, bool WIDE>
__global__ void __launch_bounds__(kRowThreads) read_kernel(const __grid_constant__ ReadArg a) {
    griddep_wait();
    const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens;
    const int nt = (int)(a.tokens - t0 < a.block_tokens ? a.tokens - t0 : a.block_tokens);
    const int h0 = blockIdx.y * a.block_heads;
    const int nh = a.heads - h0 < a.block_heads ? a.heads - h0 : a.block_heads;
    const int c = threadIdx.x;
    for (int idx = threadIdx.y; idx < nt * nh; idx += blockDim.y) {
        const int tl = idx / nh;
        const int64_t t = t0 + tl;
        int h = h0 + idx - tl * nh;
        const bool is_v = !a.has_k || h >= a.cache.kv_heads;
        if (a.has_k && is_v) h -= a.cache.kv_heads;
        const int slot = a.slots[t];
        float x[16];
        if (slot < 0 || slot >= a.cache.n_pages * kKvPage) {
            const float fill = slot < 0 ? 0.f : __uint_as_float(0x7FC00000u);
            if (slot >= 0 && a.status) atomicOr(a.status, WICI_BAD_SLOT);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = fill;
        } else {
            const uint8_t *block = a.cache.data + (int64_t)(slot / kKvPage) * a.cache.page_stride +
                                   (int64_t)(is_v ? a.cache.kv_heads + h : h) *
                                       (FMT == WICI_KV_BF16 ? kKvPage * D * 2 : kKvPage * (D + 4));
            const int place = slot & (kKvPage - 1);
            if (FMT == WICI_KV_BF16) {
                const __nv_bfloat16 *src = (const __nv_bfloat16 *)block + place * D + 16 * c;
                load8<__nv_bfloat16, true>(src, 8, x);
                load8<__nv_bfloat16, true>(src + 8, 8, x + 8);
            } else {
                const uint4 w = *(const uint4 *)(block + place * D + 16 * c);
                const float scale = ((const float *)(block + kKvPage * D))[place];
                const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 f = __half22float2(decode2<FMT>(word[j / 2] >> (16 * (j & 1))));
                    x[2 * j] = f.x * scale;
                    x[2 * j + 1] = f.y * scale;
                }
            }
        }
        T *dst = (is_v ? a.v : a.k).template row<T>(t, h) + 16 * c;
        store8<T, WIDE>(dst, 8, x);
        store8<T, WIDE>(dst + 8, 8, x + 8);
    }
}

DeviceTable<int> g_sms;

int sm_count(int *n) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
        e = g_sms.get(dev, n, [dev](int *d) { return cudaDeviceGetAttribute(d, cudaDevAttrMultiProcessorCount, dev); });
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "SM count: %s", cudaGetErrorString(e));
}

template <typename T, int FMT>
cudaError_t launch_rows(const RowsArg &a, const RowSplit &s, bool wide, cudaStream_t st) {
    const dim3 block(a.chunks, kRowThreads / a.chunks);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)s.token_blocks, s.head_blocks);
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = a.positions ? (size_t)s.tokens * 4 * a.rot_chunks * sizeof(float4) : 0;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return wide ? cudaLaunchKernelEx(&cfg, rows_kernel<T, FMT, true>, a)
                : cudaLaunchKernelEx(&cfg, rows_kernel<T, FMT, false>, a);
}

template <int FMT>
cudaError_t launch_rows(int dtype, const RowsArg &a, const RowSplit &s, bool wide, cudaStream_t st) {
    switch (dtype) {
        case WICI_BF16: return launch_rows<__nv_bfloat16, FMT>(a, s, wide, st);
        case WICI_F16: return launch_rows<__half, FMT>(a, s, wide, st);
        default: return launch_rows<float, FMT>(a, s, wide, st);
    }
}

void set_rope(RowsArg *a, const wici_rope_plan *plan, bool inverse) {
    for (int i = 0; i < 128; ++i) a->rope.turns[i] = plan->turns[i];
    a->rope.gain = plan->gain;
    a->rope.sign = inverse ? -1.f : 1.f;
    a->rope.head_dim = plan->head_dim;
    a->rope.rot = plan->rot_dim;
    a->rope.interleaved = plan->interleaved;
    a->rot_chunks = (plan->rot_dim / 2 + 7) / 8;
    a->chunks = a->rot_chunks + (plan->head_dim - plan->rot_dim + 15) / 16;
}

constexpr int64_t kMaxTokens = (int64_t)1 << 31;   // exclusive: token blocks fit a grid

template <typename T, int FMT, int D>
cudaError_t launch_read(const ReadArg &a, const RowSplit &s, bool wide, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)s.token_blocks, s.head_blocks);
    cfg.blockDim = dim3(D / 16, kRowThreads / (D / 16));
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return wide ? cudaLaunchKernelEx(&cfg, read_kernel<T, FMT, D, true>, a)
                : cudaLaunchKernelEx(&cfg, read_kernel<T, FMT, D, false>, a);
}

template <typename T, int FMT>
cudaError_t launch_read(int d, const ReadArg &a, const RowSplit &s, bool wide, cudaStream_t st) {
    return d == 64 ? launch_read<T, FMT, 64>(a, s, wide, st) : launch_read<T, FMT, 128>(a, s, wide, st);
}

template <typename T>
cudaError_t launch_read(int fmt, int d, const ReadArg &a, const RowSplit &s, bool wide, cudaStream_t st) {
    switch (fmt) {
        case WICI_KV_BF16: return launch_read<T, WICI_KV_BF16>(d, a, s, wide, st);
        case WICI_KV_INT8: return launch_read<T, WICI_KV_INT8>(d, a, s, wide, st);
        default: return launch_read<T, WICI_KV_E4M3>(d, a, s, wide, st);
    }
}

}  // namespace

extern "C" {

int wici_rope_make_plan(const wici_rope_spec *s, wici_rope_plan *plan) {
    if (!s || !plan) return fail(WICI_E_ARG, "rope: null argument");
    if (s->head_dim < 2 || s->head_dim > 256 || s->head_dim % 2)
        return fail(WICI_E_ARG, "rope: head_dim must be even and in [2, 256], got %d", s->head_dim);
    if (s->rot_dim < 2 || s->rot_dim > s->head_dim || s->rot_dim % 2)
        return fail(WICI_E_ARG, "rope: rot_dim must be even and in [2, head_dim], got %d", s->rot_dim);
    if (s->interleaved != 0 && s->interleaved != 1) return fail(WICI_E_ARG, "rope: interleaved must be 0 or 1");
    if (s->scaling < WICI_ROPE_NONE || s->scaling > WICI_ROPE_YARN) return fail(WICI_E_ARG, "rope: scaling");
    if (!(s->theta > 1.0) || !isfinite(s->theta)) return fail(WICI_E_ARG, "rope: theta must be > 1");
    if (!(s->factor >= 1.0) || !isfinite(s->factor)) return fail(WICI_E_ARG, "rope: factor must be >= 1");
    if (s->scaling == WICI_ROPE_NONE && s->factor != 1.0)
        return fail(WICI_E_ARG, "rope: a factor without a scaling rule");
    if (!(s->gain >= 0.0) || !isfinite((float)s->gain)) return fail(WICI_E_ARG, "rope: gain must be >= 0");
    const bool ranged = s->scaling == WICI_ROPE_BANDS || s->scaling == WICI_ROPE_YARN;
    if (ranged && (!(s->low > 0.0) || !(s->high > s->low) || !isfinite(s->high) || s->original_len < 1))
        return fail(WICI_E_ARG, "rope: 0 < low < high and original_len >= 1 required");
    const double two_pi = 6.283185307179586476925286766559, rot = s->rot_dim;
    double lo = 0.0, hi = 0.0, gain = s->gain;
    if (s->scaling == WICI_ROPE_YARN) {
        const double per = 2.0 * log(s->theta);
        lo = floor(rot * log(s->original_len / (s->high * two_pi)) / per);
        hi = ceil(rot * log(s->original_len / (s->low * two_pi)) / per);
        lo = lo < 0.0 ? 0.0 : lo;
        hi = hi > rot - 1.0 ? rot - 1.0 : hi;
    }
    if (gain == 0.0) gain = s->scaling == WICI_ROPE_YARN ? 0.1 * log(s->factor) + 1.0 : 1.0;
    for (int i = 0; i < 128; ++i) {
        plan->turns[i] = 0;
        if (i >= s->rot_dim / 2) continue;
        double f = pow(s->theta, -2.0 * i / rot);
        if (s->scaling == WICI_ROPE_LINEAR) {
            f /= s->factor;
        } else if (s->scaling == WICI_ROPE_BANDS) {
            double mix = (s->original_len * f / two_pi - s->low) / (s->high - s->low);
            mix = mix < 0.0 ? 0.0 : mix > 1.0 ? 1.0 : mix;
            f *= (1.0 - mix) / s->factor + mix;
        } else if (s->scaling == WICI_ROPE_YARN) {
            const double width = hi - lo > 1e-3 ? hi - lo : 1e-3;
            double r = (i - lo) / width;
            r = r < 0.0 ? 0.0 : r > 1.0 ? 1.0 : r;
            f *= (1.0 - r) + r / s->factor;
        }
        plan->turns[i] = (uint64_t)llrint(ldexp(f / two_pi, 63)) << 1;   // f <= 1: below a sixth of a turn
    }
    plan->gain = (float)gain;
    plan->head_dim = s->head_dim;
    plan->rot_dim = s->rot_dim;
    plan->interleaved = s->interleaved;
    return WICI_OK;
}

int wici_rope(void *cuda_stream, const wici_rope_plan *plan, int32_t inverse, const int32_t *positions,
              int64_t tokens, const wici_heads *x, const wici_heads *y) {
    if (const char *m = check_rope(plan)) return fail(WICI_E_ARG, "rope: %s", m);
    if (inverse != 0 && inverse != 1) return fail(WICI_E_ARG, "rope: inverse must be 0 or 1");
    if (tokens < 0 || tokens >= kMaxTokens) return fail(WICI_E_ARG, "rope: tokens must be in [0, 2^31)");
    if (const char *m = check_heads(x, tokens, plan->head_dim, false)) return fail(WICI_E_ARG, "rope x: %s", m);
    if (const char *m = check_heads(y, tokens, plan->head_dim, true)) return fail(WICI_E_ARG, "rope y: %s", m);
    if (x->dtype != y->dtype || x->heads != y->heads) return fail(WICI_E_ARG, "rope: x and y differ in type or heads");
    if (tokens == 0) return WICI_OK;
    if (!positions) return fail(WICI_E_ARG, "rope: null positions");
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    RowsArg a = {};
    set_rope(&a, plan, inverse == 1);
    a.q = heads_arg(x);
    a.q_out = heads_arg(y);
    a.positions = positions;
    a.tokens = tokens;
    a.q_heads = a.heads = x->heads;
    const RowSplit s = split_rows(tokens, a.heads, kRowThreads / a.chunks, kBlockTokens, 8 * sms);
    a.block_tokens = s.tokens;
    a.block_heads = s.heads;
    const bool wide = wide_heads(x) && wide_heads(y) && plan->rot_dim % 16 == 0 && plan->head_dim % 8 == 0;
    const cudaError_t e = launch_rows<kRopeOnly>(x->dtype, a, s, wide, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "rope: %s", cudaGetErrorString(e));
}

int64_t wici_kv_page_bytes(int32_t format, int32_t n_kv_heads, int32_t head_dim) {
    if ((format != WICI_KV_BF16 && format != WICI_KV_INT8 && format != WICI_KV_E4M3) ||
        (head_dim != 64 && head_dim != 128) || n_kv_heads < 1)
        return 0;
    return 2 * (int64_t)n_kv_heads * kv_block_bytes(format, head_dim);
}

int wici_kv_append(void *cuda_stream, const wici_kv_cache *cache, const int32_t *slots, int64_t tokens,
                   const wici_heads *k, const wici_heads *v, const wici_rope_plan *rope, const int32_t *positions,
                   const wici_heads *q, const wici_heads *q_out, int32_t *status) {
    if (const char *m = check_cache(cache)) return fail(WICI_E_ARG, "append: %s", m);
    if (tokens < 0 || tokens >= kMaxTokens) return fail(WICI_E_ARG, "append: tokens must be in [0, 2^31)");
    const int d = cache->head_dim;
    if (const char *m = check_heads(k, tokens, d, false)) return fail(WICI_E_ARG, "append k: %s", m);
    if (const char *m = check_heads(v, tokens, d, false)) return fail(WICI_E_ARG, "append v: %s", m);
    if (k->heads != cache->n_kv_heads || v->heads != cache->n_kv_heads || k->dtype != v->dtype)
        return fail(WICI_E_ARG, "append: k and v need the cache's heads and one type");
    if (!q != !q_out) return fail(WICI_E_ARG, "append: q and q_out come together");
    if (rope) {
        if (const char *m = check_rope(rope)) return fail(WICI_E_ARG, "append: %s", m);
        if (rope->head_dim != d || rope->rot_dim % 16)
            return fail(WICI_E_ARG, "append: the rope needs the cache's head_dim and a rot_dim that is a multiple of 16");
    } else if (q || positions) {
        return fail(WICI_E_ARG, "append: positions and q come with a rope");
    }
    if (q) {
        if (const char *m = check_heads(q, tokens, d, false)) return fail(WICI_E_ARG, "append q: %s", m);
        if (const char *m = check_heads(q_out, tokens, d, true)) return fail(WICI_E_ARG, "append q_out: %s", m);
        if (q->heads != q_out->heads || q->dtype != k->dtype || q_out->dtype != k->dtype)
            return fail(WICI_E_ARG, "append: q and q_out need the same heads and k's type");
    }
    if (tokens == 0) return WICI_OK;
    if (!slots || (rope && !positions)) return fail(WICI_E_ARG, "append: null slots or positions");
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    RowsArg a = {};
    a.rope.rot = 0;
    a.chunks = d / 16;
    if (rope) set_rope(&a, rope, false);
    a.rotate_k = rope != nullptr;
    a.q = heads_arg(q);
    a.q_out = heads_arg(q_out);
    a.k = heads_arg(k);
    a.v = heads_arg(v);
    a.cache = cache_arg(cache);
    a.positions = positions;
    a.slots = slots;
    a.status = status;
    a.tokens = tokens;
    a.q_heads = q ? q->heads : 0;
    a.heads = a.q_heads + 2 * cache->n_kv_heads;
    const RowSplit s = split_rows(tokens, a.heads, kRowThreads / a.chunks, kBlockTokens, 8 * sms);
    a.block_tokens = s.tokens;
    a.block_heads = s.heads;
    const bool wide = wide_heads(k) && wide_heads(v) && (!q || (wide_heads(q) && wide_heads(q_out)));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    switch (cache->format) {
        case WICI_KV_BF16: e = launch_rows<WICI_KV_BF16>(k->dtype, a, s, wide, st); break;
        case WICI_KV_INT8: e = launch_rows<WICI_KV_INT8>(k->dtype, a, s, wide, st); break;
        default: e = launch_rows<WICI_KV_E4M3>(k->dtype, a, s, wide, st); break;
    }
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "append: %s", cudaGetErrorString(e));
}

int wici_kv_read(void *cuda_stream, const wici_kv_cache *cache, const int32_t *slots, int64_t tokens,
                 const wici_heads *k, const wici_heads *v, int32_t *status) {
    if (const char *m = check_cache(cache)) return fail(WICI_E_ARG, "read: %s", m);
    if (tokens < 0 || tokens >= kMaxTokens) return fail(WICI_E_ARG, "read: tokens must be in [0, 2^31)");
    if (!k && !v) return fail(WICI_E_ARG, "read: neither k nor v");
    const int d = cache->head_dim;
    for (const wici_heads *t : {k, v}) {
        if (!t) continue;
        if (const char *m = check_heads(t, tokens, d, true)) return fail(WICI_E_ARG, "read: %s", m);
        if (t->heads != cache->n_kv_heads) return fail(WICI_E_ARG, "read: k and v need the cache's heads");
    }
    if (k && v && k->dtype != v->dtype) return fail(WICI_E_ARG, "read: k and v need one type");
    if (tokens == 0) return WICI_OK;
    if (!slots) return fail(WICI_E_ARG, "read: null slots");
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    ReadArg a = {};
    a.k = heads_arg(k);
    a.v = heads_arg(v);
    a.cache = cache_arg(cache);
    a.slots = slots;
    a.status = status;
    a.tokens = tokens;
    a.heads = cache->n_kv_heads * ((k ? 1 : 0) + (v ? 1 : 0));
    a.has_k = k != nullptr;
    const RowSplit s = split_rows(tokens, a.heads, kRowThreads / (d / 16), 1 << 16, 8 * sms);
    a.block_tokens = s.tokens;
    a.block_heads = s.heads;
    const bool wide = (!k || wide_heads(k)) && (!v || wide_heads(v));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    switch ((k ? k : v)->dtype) {
        case WICI_BF16: e = launch_read<__nv_bfloat16>(cache->format, d, a, s, wide, st); break;
        case WICI_F16: e = launch_read<__half>(cache->format, d, a, s, wide, st); break;
        default: e = launch_read<float>(cache->format, d, a, s, wide, st); break;
    }
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "read: %s", cudaGetErrorString(e));
}

}  // extern "C"
