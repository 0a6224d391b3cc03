// Rotary positions, and writing and reading a paged key-value cache (include/wici_ops.h).
//
// The three are row-wise: a row is one head of one token, cut into chunks of 16 elements, one
// lane each.  All are bound by HBM (each element is read and written once; a rotation is 6
// operations a pair, a quantisation 3 an element), and by launch latency when the call is a step
// of few tokens.  Measured (device time): rotation of 8192 tokens of 40 heads of 128 in bf16
// 28.3 us, 5.9 TB/s (a copy of that size: 6.4); append of 16384 tokens, 32 q heads rotated, 8 k
// and v heads to e4m3, 69.1 us, 5.4 TB/s, of which its arithmetic is 3 us; read of 30011 tokens from
// e4m3 to bf16 32.1 us, 5.8 TB/s; one token of a step 2.3 to 3.4 us.  From and to e2m1: append of 16384 tokens, 8 k and v
// heads in bf16, nothing rotated, 22.1 us, 3.9 TB/s: issue slots 68% busy, stalls of fixed latencies and of loads alike; with
// rotated keys 38.2 us, with 32 q heads too 76; read of 30011 tokens to bf16 28.8 us, 5.6 TB/s.
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

constexpr int kRopeOnly = -1;         // FMT of a launch without a cache
enum Path { WIDE_HALF, WIDE_PAIRS, WIDE_PLAIN, NARROW };   // 16-byte accesses of either layout or without a rope, or element by element

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
    int block_tokens;                 // a power of two
    int q_heads, heads;               // rows of a token: q heads, then (with a cache) k heads and v heads
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

// the largest of three, NaN where one is
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The largest magnitudes of the two blocks of 16 elements that a lane's two groups of 8 (with `own` as theirs) lie in.  Where halves of a row
// are rotated, the other 8 of a block are another lane's: group c of the row's rotated part is lane c's first one, group
// rot_chunks + c its second.
__device__ __forceinline__ void blocks_of_16(const float *own, bool halves, const RowsArg &a, float *most) {
    if (!a.rotate_k || a.rope.interleaved) {       // the same for every lane
        most[0] = most[1] = max3(own[0], own[1], 0.f);
        return;
    }
    const int c = threadIdx.x, first = (threadIdx.y * blockDim.x & 31);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int other = (c + i * a.rot_chunks) ^ 1;
        const bool second = other >= a.rot_chunks;
        const int from = halves ? first + other - (second ? a.rot_chunks : 0) : first + c;
        const float u = __shfl_sync(0xffffffffu, own[0], from), v = __shfl_sync(0xffffffffu, own[1], from);
        most[i] = max3(own[i], halves ? second ? v : u : own[1 - i], 0.f);
    }
}

// One launch rotates q rows (FMT = kRopeOnly: all rows) and writes k and v rows into the cache.
// A block takes block_tokens tokens.  It computes their cosines and sines once, one pair a thread
// and turn, through shared memory; then a thread keeps its token, with its chunk's cosines and
// sines in registers, and walks over the token's heads: what is left for a row is its loads (issued
// before the row ahead of it is worked on), the arithmetic and its stores.  Lanes of a warp take
// neighbouring heads of a token: a packed row's heads lie side by side.  (e2m1 has 80 registers in place of 64, where rotated
// rows spill: 8 k and v heads in fp32 rotated, 1251 tokens of 64 5.6 us, 6.3 with 64, 16384 of 128 38.6 and 41.8; not
// rotated, in bf16, 22.1 and 21.5.)
template <typename T, int FMT, int PATH>
__global__ void __launch_bounds__(kRowThreads, FMT == WICI_KV_E2M1 ? 6 : kRowBlocks) rows_kernel(const __grid_constant__ RowsArg a) {
    constexpr bool WIDE = PATH != NARROW, PLAIN = PATH == WIDE_PLAIN;
    constexpr int W = sizeof(T) / 2;                             // 16-byte words of 8 elements
    extern __shared__ float4 cs[];    // [token][4][rot_chunks]: (cos, sin) of pairs 8 chunk + 2 j, + 2 j + 1
    const bool pairs = PATH == NARROW ? a.rope.interleaved : PATH == WIDE_PAIRS;
    const int c = threadIdx.x, half = a.rope.rot / 2;
    const int tid = threadIdx.y * blockDim.x + c, nthreads = blockDim.x * blockDim.y;
    // The chunk's two groups of 8 elements in a rotated row: where they start, how many they hold.  Interleaved
    // rows are cut as they lie, so a chunk may hold pairs that are not rotated; halves are cut apart.
    int o0, o1, n0, n1;
    const bool turns = !PLAIN && c < a.rot_chunks;
    if (turns && !pairs) {
        o0 = 8 * c;
        o1 = half + 8 * c;
        n0 = n1 = half - 8 * c < 8 ? half - 8 * c : 8;
    } else {
        o0 = pairs || PLAIN ? 16 * c : a.rope.rot + 16 * (c - a.rot_chunks);
        o1 = o0 + 8;
        const int n = PLAIN ? 16 : a.rope.head_dim - o0 < 16 ? a.rope.head_dim - o0 : 16;
        n0 = n < 8 ? n : 8;
        n1 = n - n0;
    }
    griddep_launch_dependents();
    griddep_wait();
    const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens;
    const int step = blockDim.y / a.block_tokens, tl = threadIdx.y / step;
    const int64_t t = t0 + tl < a.tokens ? t0 + tl : a.tokens - 1;   // past the end: the last token's, not stored
    const bool here = t0 + tl < a.tokens;
    int slot = FMT != kRopeOnly && here ? a.slots[t] : -1;
    const T *const sq = a.q.template row<T>(t, 0), *const sk = a.k.template row<T>(t, 0), *const sv = a.v.template row<T>(t, 0);
    T *const dq = a.q_out.template row<T>(t, 0);
    const int k0 = a.q_heads, v0 = FMT == kRopeOnly ? a.heads : a.q_heads + a.cache.kv_heads;   // first k row, first v row
    // a row's two groups of elements as they stand
    auto fetch = [&](int h, uint4 *raw) {
        const bool is_q = !PLAIN && (FMT == kRopeOnly || h < k0), is_v = !is_q && h >= v0, rotate = !PLAIN && (is_q || (!is_v && a.rotate_k));
        const T *src = is_q ? sq + h * a.q.hs : is_v ? sv + (h - v0) * a.v.hs : sk + (h - k0) * a.k.hs;
        const T *p0 = src + (rotate ? o0 : 16 * c), *p1 = src + (rotate ? o1 : 16 * c + 8);
        if (WIDE) {
#pragma unroll
            for (int i = 0; i < W; ++i) raw[i] = ((const uint4 *)p0)[i];
            if (FMT != kRopeOnly || n1 > 0) {
#pragma unroll
                for (int i = 0; i < W; ++i) raw[W + i] = ((const uint4 *)p1)[i];
            }
        } else {
            float *x = (float *)raw;
            load8(p0, rotate ? n0 : 8, x);
            load8(p1, rotate ? n1 : 8, x + 8);
        }
    };
    constexpr int RAW = WIDE ? 2 * W : 4;
    uint4 raw[RAW] = {};
    const int h0 = threadIdx.y % step;
    if (h0 < a.heads) fetch(h0, raw);     // on its way while the angles are computed
    float2 w[8];                                                 // cosine and sine of the chunk's pairs
    if (!PLAIN && a.positions) {
        const int per = 8 * a.rot_chunks;
        for (int i = tid; i < a.block_tokens * per; i += nthreads) {
            const int tt = i / per, p = i - tt * per;
            const int64_t token = t0 + tt < a.tokens ? t0 + tt : a.tokens - 1;
            float2 v = make_float2(1.f, 0.f);
            if (p < half) {
                v = turn_of((uint64_t)(int64_t)a.positions[token] * a.rope.turns[p]);
                v.x *= a.rope.gain;
                v.y *= a.rope.gain * a.rope.sign;
            }
            ((float2 *)cs)[(((tt * 4 + (p & 7) / 2) * a.rot_chunks + p / 8) << 1) + (p & 1)] = v;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float4 v = cs[(tl * 4 + j) * a.rot_chunks + (turns ? c : 0)];
            w[2 * j] = make_float2(v.x, v.y);
            w[2 * j + 1] = make_float2(v.z, v.w);
        }
    }
    if (FMT != kRopeOnly && slot >= a.cache.n_pages * kKvPage) {
        if (a.status) atomicOr(a.status, WICI_BAD_SLOT);
        slot = -1;
    }
    const int d = FMT == kRopeOnly ? 0 : 16 * a.chunks, where = slot & (kKvPage - 1);
    const int kv_block = FMT == kRopeOnly ? 0 : kv_block_bytes(FMT, d);
    uint8_t *page = FMT == kRopeOnly || slot < 0 ? nullptr : a.cache.data + (int64_t)(slot / kKvPage) * a.cache.page_stride;
    // every lane of a warp stays: rows are reduced by shuffles
    for (int base = 0; base < a.heads; base += step) {
        const int h = base + h0;
        const bool live = here && h < a.heads;
        const bool is_q = !PLAIN && (FMT == kRopeOnly || h < k0), is_v = !is_q && h >= v0, rotate = !PLAIN && (is_q || (!is_v && a.rotate_k));
        float x[16];
        if (WIDE) {
            const T *e = (const T *)raw;
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = to_f32(e[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = ((const float *)raw)[j];
        }
        if (h + step < a.heads) fetch(h + step, raw);
        const int p0 = rotate ? o0 : 16 * c, p1 = rotate ? o1 : 16 * c + 8;
        if (rotate && turns) {
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                const float xa = pairs ? x[2 * p] : x[p], xb = pairs ? x[2 * p + 1] : x[p + 8];
                const float ya = xa * w[p].x - xb * w[p].y, yb = xa * w[p].y + xb * w[p].x;
                // the pair's own places are read and written by this step alone
                if (pairs) {
                    if (8 * c + p < half) x[2 * p] = ya, x[2 * p + 1] = yb;
                } else {
                    x[p] = ya, x[p + 8] = yb;
                }
            }
        }
        if (is_q) {
            if (live) {
                T *dst = dq + h * a.q_out.hs;
                store8<T, WIDE>(dst + p0, n0, x);
                if (n1 > 0) store8<T, WIDE>(dst + p1, n1, x + 8);
            }
            if (FMT == kRopeOnly || FMT == WICI_KV_BF16) continue;
        }
        if (FMT != kRopeOnly) {
            uint8_t *block = page + (int64_t)(h - k0) * kv_block;   // V's blocks follow K's
            const bool store = live && !is_q && slot >= 0;
            if (FMT == WICI_KV_BF16) {
                if (store) {
                    __nv_bfloat16 *dst = (__nv_bfloat16 *)block + where * d;
                    store8<__nv_bfloat16, true>(dst + p0, 8, x);
                    store8<__nv_bfloat16, true>(dst + p1, 8, x + 8);
                }
            } else if (__any_sync(0xffffffffu, store)) {
                // the row's largest magnitude
                float top, own[2];
                if (FMT == WICI_KV_E2M1) {                           // from its groups of 8
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        own[i] = fabsf(x[8 * i]);
#pragma unroll
                        for (int j = 1; j < 7; j += 2) own[i] = max3(own[i], fabsf(x[8 * i + j]), fabsf(x[8 * i + j + 1]));
                        own[i] = max3(own[i], fabsf(x[8 * i + 7]), 0.f);
                    }
                    top = max3(own[0], own[1], 0.f);
                } else {
                    top = fabsf(x[0]);
#pragma unroll
                    for (int j = 1; j < 15; j += 2) top = max3(top, fabsf(x[j]), fabsf(x[j + 1]));
                    top = max3(top, fabsf(x[15]), 0.f);
                }
                for (int o = a.chunks / 2; o > 0; o >>= 1) top = max3(top, __shfl_xor_sync(0xffffffffu, top, o), 0.f);
                if (FMT == WICI_KV_E2M1) {
                    float most[2];
                    if (PLAIN) most[0] = most[1] = max3(own[0], own[1], 0.f);
                    else blocks_of_16(own, rotate && turns && !pairs, a, most);
                    if (store) {
                        constexpr float kPer = 1.f / kE2m1Top;     // the quotient, right to its last bit
                        const float near = top * kPer, s = fmaf(fmaf(-near, kE2m1Top, top), kPer, near);
                        const bool finite = top < __uint_as_float(kInfBits), some = finite && s >= kE2m1Least;
                        const float per6 = reciprocal(6.f * s);
                        // given 16-bit values, not rotated ones: one conversion each
                        const float left = fmaf(-s, kE2m1Top, top), nudge = nudge_of(left);
                        const bool sure = sizeof(T) == 2 && !rotate && left != 0.f;
                        uint8_t *row = block + where * (d / 2), *each = block + kKvPage * (d / 2) + where * (d / 16);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int p = i ? p1 : p0;
                            uint32_t b = 0, codes = 0;
                            if (some && sure) {
                                b = __nv_cvt_float_to_fp8(most[i] * (per6 * nudge), __NV_SATFINITE, __NV_E4M3);
                                const float unit = e4m3_value(b) * s;
                                codes = encode_e2m1(x + 8 * i, unit > 0.f ? reciprocal(unit) * nudge : 0.f);
                            } else if (some) {
                                b = block_scale(most[i], s, per6);
                                codes = quantise_e2m1(x + 8 * i, e4m3_value(b), s);
                            }
                            *(uint32_t *)(row + p / 2) = codes;
                            if ((p & 8) == 0) each[p / 16] = (uint8_t)b;
                        }
                        if (c == 0)
                            ((float *)(block + kv_scales_at(FMT, d)))[where] = finite ? some ? s : 0.f : __uint_as_float(0x7FC00000u);
                    }
                } else if (store) {
                    uint32_t code[4];
                    const float scale = quantise16<FMT>(x, top, code);
                    uint8_t *dst = block + where * d;
                    *(uint2 *)(dst + p0) = make_uint2(code[0], code[1]);
                    *(uint2 *)(dst + p1) = make_uint2(code[2], code[3]);
                    if (c == 0) ((float *)(block + kKvPage * d))[where] = scale;
                }
            }
        }
    }
}

// Rotation of halves that do not lie in whole groups of 8 elements (rot_dim no multiple of 16): an element's
// partner, rot_dim / 2 places on or back, starts anywhere in a 16-byte word.  Element by element that costs as many
// accesses as elements; so a lane takes whole words, the row's words pass through the warp's shared memory, and a
// lane cuts its word's partners out of the two words that hold them.  A row is read before any of it is written:
// y may be x.  8192 tokens of 32 heads of 128, 126 of them rotated, in bf16: 33.8 us, 4.0 TB/s, bound by the
// instructions of the cut (90.7 element by element; 23.2 where all 128 turn, in rows_kernel); 100 of them rotated,
// in fp32: 44.4 to 46.5 us, 6 TB/s (with one word a lane 57.5).
constexpr int kRaggedTokens = 4;      // tokens of a block at most: a warp keeps to one
constexpr int kWarps = kRowThreads / 32;

template <typename T>
__global__ void __launch_bounds__(kRowThreads, kRowBlocks) ragged_kernel(const __grid_constant__ RowsArg a) {
    constexpr int E = 16 / sizeof(T);              // elements of a word
    constexpr int NW = sizeof(T) / 2;              // words of a lane: 8 elements of either size
    __shared__ uint4 stage[kWarps][32 * NW];
    __shared__ float2 cs[kRaggedTokens][128];
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, half = a.rope.rot / 2;
    const int words = a.rope.head_dim / E, lanes = (words + NW - 1) / NW, rows = 32 / lanes;
    const int sub = lane / lanes, c = lane - sub * lanes;
    griddep_launch_dependents();
    griddep_wait();
    const int per = kWarps / a.block_tokens, tl = warp / per, step = per * rows;
    const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens;
    const int64_t t = t0 + tl < a.tokens ? t0 + tl : a.tokens - 1;   // past the end: the last token's, not stored
    const bool here = t0 + tl < a.tokens && sub < rows;
    const T *const src = a.q.template row<T>(t, 0);
    T *const dst = a.q_out.template row<T>(t, 0);
    uint4 raw[NW] = {};
    auto fetch = [&](int h) {
#pragma unroll
        for (int i = 0; i < NW; ++i)
            if (here && h < a.heads && c + i * lanes < words) raw[i] = ((const uint4 *)(src + h * a.q.hs))[c + i * lanes];
    };
    const int h0 = (warp - tl * per) * rows + sub;
    fetch(h0);
    for (int i = threadIdx.x; i < a.block_tokens * half; i += kRowThreads) {
        const int tt = i / half, p = i - tt * half;
        const int64_t token = t0 + tt < a.tokens ? t0 + tt : a.tokens - 1;
        const float2 v = turn_of((uint64_t)(int64_t)a.positions[token] * a.rope.turns[p]);
        cs[tt][p] = make_float2(v.x * a.rope.gain, v.y * a.rope.gain * a.rope.sign);
    }
    __syncthreads();
    float2 w[NW * E];                              // an element's cosine, and the sine that its partner takes
#pragma unroll
    for (int j = 0; j < NW * E; ++j) {
        const int e = (c + j / E * lanes) * E + j % E;
        w[j] = cs[tl][e < half ? e : e < 2 * half ? e - half : 0];
        if (e < half) w[j].y = -w[j].y;
    }
    uint4 *const row = stage[warp] + (sub < rows ? sub * words : 0);
    // E elements from element q of the row on, those outside the row anything
    auto cut = [&](int q, T *x) {
        const int at = q >= 0 ? q / E : (q - E + 1) / E, bytes = (q - at * E) * (int)sizeof(T);
        alignas(16) uint32_t r[8];
        *(uint4 *)r = row[at < 0 ? 0 : at < words ? at : words - 1];
        *(uint4 *)(r + 4) = row[at + 1 < 0 ? 0 : at + 1 < words ? at + 1 : words - 1];
#pragma unroll
        for (int i = 0; i < 6; ++i) r[i] = bytes & 8 ? r[i + 2] : r[i];
#pragma unroll
        for (int i = 0; i < 5; ++i) r[i] = bytes & 4 ? r[i + 1] : r[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) ((uint32_t *)x)[i] = __funnelshift_r(r[i], r[i + 1], bytes & 2 ? 16 : 0);
    };
    for (int base = 0; base < a.heads; base += step) {
        const int h = base + h0;
        alignas(16) T own[NW * E];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            ((uint4 *)own)[i] = raw[i];
            if (sub < rows && c + i * lanes < words) row[c + i * lanes] = raw[i];
        }
        __syncwarp();
        fetch(h + step);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int e0 = (c + i * lanes) * E;
            alignas(16) T other[E];
            cut(e0 < half ? e0 + half : e0 - half, other);
            if (e0 < half && e0 + E > half) {      // both halves meet in this word
                alignas(16) T back[E];
                cut(e0 - half, back);
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (e0 + j >= half) other[j] = back[j];
            }
            float y[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float x = to_f32(own[i * E + j]);
                y[j] = e0 + j < 2 * half ? x * w[i * E + j].x + to_f32(other[j]) * w[i * E + j].y : x;
            }
            if (here && h < a.heads && e0 < a.rope.head_dim) {
                alignas(16) T out[E];
#pragma unroll
                for (int j = 0; j < E; ++j) from_f32(y[j], out[j]);
                *(uint4 *)(dst + h * a.q_out.hs + e0) = *(const uint4 *)out;
            }
        }
        __syncwarp();                              // the row has been read
    }
}

struct ReadArg {
    HeadsArg k, v;
    CacheArg cache;
    const int32_t *slots;
    int32_t *status;
    int64_t tokens;
    int block_tokens;                 // a power of two
    int heads;                        // rows of a token: those of k, then those of v
    bool has_k;
};

// Rows of the cache to rows of k and v.  A thread keeps its token and walks over the heads, kReadRows
// of them under way at a time; a warp reads the same head of up to four tokens: side by side in a page.
constexpr int kReadRows = 4;
template <typename T, int FMT, int D, bool WIDE>
__global__ void __launch_bounds__(kRowThreads, kRowBlocks) read_kernel(const __grid_constant__ ReadArg a) {
    constexpr int W = FMT == WICI_KV_BF16 ? 2 : 1;               // 16-byte words of a lane's 16 values
    constexpr int kBlock = kv_block_bytes(FMT, D);
    griddep_launch_dependents();
    griddep_wait();
    const int64_t t = (int64_t)blockIdx.x * a.block_tokens + (threadIdx.y & (a.block_tokens - 1));
    if (t >= a.tokens) return;
    const int c = threadIdx.x, step = blockDim.y / a.block_tokens;
    const int slot = a.slots[t], where = slot & (kKvPage - 1);
    const bool good = slot >= 0 && slot < a.cache.n_pages * kKvPage;
    // no slot: zeros; a slot outside the cache: NaN
    const float fill = slot < 0 ? 0.f : __uint_as_float(0x7FC00000u);
    if (!good && slot >= 0 && a.status) atomicOr(a.status, WICI_BAD_SLOT);
    const uint8_t *src = a.cache.data + (int64_t)(good ? slot / kKvPage : 0) * a.cache.page_stride;
    if (!a.has_k) src += a.cache.kv_heads * (int64_t)kBlock;
    T *const dk = a.k.template row<T>(t, 0) + 16 * c, *const dv = a.v.template row<T>(t, 0) + 16 * c;
    for (int h0 = threadIdx.y / a.block_tokens; h0 < a.heads; h0 += kReadRows * step) {
        uint4 word[kReadRows][W];
        float scale[kReadRows];
#pragma unroll
        for (int i = 0; i < kReadRows; ++i) {
            const int h = h0 + i * step;
            scale[i] = fill;
#pragma unroll
            for (int w = 0; w < W; ++w) word[i][w] = make_uint4(0, 0, 0, 0);
            if (good && h < a.heads) {
                const uint8_t *block = src + (int64_t)h * kBlock;
                if (FMT == WICI_KV_BF16) {
#pragma unroll
                    for (int w = 0; w < W; ++w) word[i][w] = *(const uint4 *)(block + (where * D + 16 * c) * 2 + 16 * w);
                } else if (FMT == WICI_KV_E2M1) {
                    const uint2 codes = *(const uint2 *)(block + where * (D / 2) + 8 * c);
                    word[i][0] = make_uint4(codes.x, codes.y, block[kKvPage * (D / 2) + where * (D / 16) + c], 0);
                    scale[i] = ((const float *)(block + kv_scales_at(FMT, D)))[where];
                } else {
                    word[i][0] = *(const uint4 *)(block + where * D + 16 * c);
                    scale[i] = ((const float *)(block + kKvPage * D))[where];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kReadRows; ++i) {
            const int h = h0 + i * step;
            if (h >= a.heads) break;
            float x[16];
            const uint32_t *w = (const uint32_t *)word[i];
            if (FMT == WICI_KV_BF16) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[2 * j] = good ? bf16lo(w[j]) : fill;
                    x[2 * j + 1] = good ? bf16hi(w[j]) : fill;
                }
            } else if (FMT == WICI_KV_E2M1) {
                const float b = e4m3_value(w[2]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t h[4];
                    decode_e2m1(w[j], h);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {                // code * b is exact
                        const float2 f = __half22float2(*(const __half2 *)&h[k]);
                        x[8 * j + 2 * k] = f.x * b * scale[i], x[8 * j + 2 * k + 1] = f.y * b * scale[i];
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t lo, hi;
                    decode4<FMT>(w[j], lo, hi);
                    const float2 f = __half22float2(*(const __half2 *)&lo), g = __half22float2(*(const __half2 *)&hi);
                    x[4 * j] = f.x * scale[i], x[4 * j + 1] = f.y * scale[i];
                    x[4 * j + 2] = g.x * scale[i], x[4 * j + 3] = g.y * scale[i];
                }
            }
            const bool is_v = !a.has_k || h >= a.cache.kv_heads;
            T *dst = is_v ? dv + (a.has_k ? h - a.cache.kv_heads : h) * a.v.hs : dk + h * a.k.hs;
            store8<T, WIDE>(dst, 8, x);
            store8<T, WIDE>(dst + 8, 8, x + 8);
        }
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

template <typename Kern, typename Arg>
cudaError_t launch_blocks(Kern kern, const Arg &a, dim3 block, size_t smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.tokens + a.block_tokens - 1) / a.block_tokens));
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

template <typename T, int FMT>
cudaError_t launch_rows(RowsArg &a, bool wide, int sms, cudaStream_t st) {
    const RowBlock b = row_block(a.tokens, a.heads, a.chunks, sms);
    a.block_tokens = b.tokens;
    const dim3 block(a.chunks, b.rows);
    const size_t smem = a.positions ? (size_t)b.tokens * 4 * a.rot_chunks * sizeof(float4) : 0;
    if (!wide) return launch_blocks(rows_kernel<T, FMT, NARROW>, a, block, smem, st);
    // Without a rope e2m1, where instructions count, has a kernel of its own: append of 16384 tokens 22.1 us, 29.2 where rows
    // that might turn are told apart.  The other formats are bound by HBM either way.
    if constexpr (FMT == WICI_KV_E2M1)
        if (!a.positions) return launch_blocks(rows_kernel<T, FMT, WIDE_PLAIN>, a, block, smem, st);
    return a.rope.interleaved ? launch_blocks(rows_kernel<T, FMT, WIDE_PAIRS>, a, block, smem, st)
                              : launch_blocks(rows_kernel<T, FMT, WIDE_HALF>, a, block, smem, st);
}

template <int FMT>
cudaError_t launch_rows(int dtype, RowsArg &a, bool wide, int sms, cudaStream_t st) {
    switch (dtype) {
        case WICI_BF16: return launch_rows<__nv_bfloat16, FMT>(a, wide, sms, st);
        case WICI_F16: return launch_rows<__half, FMT>(a, wide, sms, st);
        default: return launch_rows<float, FMT>(a, wide, sms, st);
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
    a->chunks = plan->interleaved ? (plan->head_dim + 15) / 16 : a->rot_chunks + (plan->head_dim - plan->rot_dim + 15) / 16;
}

constexpr int64_t kMaxTokens = (int64_t)1 << 31;   // exclusive

template <typename T, int FMT>
cudaError_t launch_read(int d, ReadArg &a, bool wide, int sms, cudaStream_t st) {
    const RowBlock b = row_block(a.tokens, a.heads, d / 16, sms);
    a.block_tokens = b.tokens;
    const dim3 block(d / 16, b.rows);
    if (d == 64)
        return wide ? launch_blocks(read_kernel<T, FMT, 64, true>, a, block, 0, st)
                    : launch_blocks(read_kernel<T, FMT, 64, false>, a, block, 0, st);
    return wide ? launch_blocks(read_kernel<T, FMT, 128, true>, a, block, 0, st)
                : launch_blocks(read_kernel<T, FMT, 128, false>, a, block, 0, st);
}

template <typename T>
cudaError_t launch_read(int fmt, int d, ReadArg &a, bool wide, int sms, cudaStream_t st) {
    switch (fmt) {
        case WICI_KV_BF16: return launch_read<T, WICI_KV_BF16>(d, a, wide, sms, st);
        case WICI_KV_INT8: return launch_read<T, WICI_KV_INT8>(d, a, wide, sms, st);
        case WICI_KV_E2M1: return launch_read<T, WICI_KV_E2M1>(d, a, wide, sms, st);
        default: return launch_read<T, WICI_KV_E4M3>(d, a, wide, sms, st);
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
    if (!positions || !words(positions)) return fail(WICI_E_ARG, "rope: positions null or unaligned");
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    RowsArg a = {};
    set_rope(&a, plan, inverse == 1);
    a.q = heads_arg(x);
    a.q_out = heads_arg(y);
    a.positions = positions;
    a.q_heads = a.heads = x->heads;
    a.tokens = tokens;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool aligned = wide_heads(x) && wide_heads(y);
    cudaError_t e;
    if (aligned && !plan->interleaved && plan->rot_dim % 16 && plan->head_dim % (16 / dtype_bytes(x->dtype)) == 0) {
        a.block_tokens = tokens_of_block(tokens, kRaggedTokens, sms);
        switch (x->dtype) {
            case WICI_BF16: e = launch_blocks(ragged_kernel<__nv_bfloat16>, a, dim3(kRowThreads), 0, st); break;
            case WICI_F16: e = launch_blocks(ragged_kernel<__half>, a, dim3(kRowThreads), 0, st); break;
            default: e = launch_blocks(ragged_kernel<float>, a, dim3(kRowThreads), 0, st); break;
        }
    } else {
        const bool wide = aligned && plan->head_dim % 8 == 0 && (plan->interleaved || plan->rot_dim % 16 == 0);
        e = launch_rows<kRopeOnly>(x->dtype, a, wide, sms, st);
    }
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "rope: %s", cudaGetErrorString(e));
}

int64_t wici_kv_page_bytes(int32_t format, int32_t n_kv_heads, int32_t head_dim) {
    if (!known_format(format) || (head_dim != 64 && head_dim != 128) || n_kv_heads < 1) return 0;
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
    if (!slots || (rope && !positions) || !words(slots) || !words(positions) || !words(status))
        return fail(WICI_E_ARG, "append: slots or positions null, or one of them or status unaligned");
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
    a.q_heads = q ? q->heads : 0;
    a.heads = a.q_heads + 2 * cache->n_kv_heads;
    a.tokens = tokens;
    const bool wide = wide_heads(k) && wide_heads(v) && (!q || (wide_heads(q) && wide_heads(q_out)));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    switch (cache->format) {
        case WICI_KV_BF16: e = launch_rows<WICI_KV_BF16>(k->dtype, a, wide, sms, st); break;
        case WICI_KV_INT8: e = launch_rows<WICI_KV_INT8>(k->dtype, a, wide, sms, st); break;
        case WICI_KV_E2M1: e = launch_rows<WICI_KV_E2M1>(k->dtype, a, wide, sms, st); break;
        default: e = launch_rows<WICI_KV_E4M3>(k->dtype, a, wide, sms, st); break;
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
    if (!slots || !words(slots) || !words(status)) return fail(WICI_E_ARG, "read: slots null, or slots or status unaligned");
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    ReadArg a = {};
    a.k = heads_arg(k);
    a.v = heads_arg(v);
    a.cache = cache_arg(cache);
    a.slots = slots;
    a.status = status;
    a.heads = cache->n_kv_heads * ((k ? 1 : 0) + (v ? 1 : 0));
    a.tokens = tokens;
    a.has_k = k != nullptr;
    const bool wide = (!k || wide_heads(k)) && (!v || wide_heads(v));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    switch ((k ? k : v)->dtype) {
        case WICI_BF16: e = launch_read<__nv_bfloat16>(cache->format, d, a, wide, sms, st); break;
        case WICI_F16: e = launch_read<__half>(cache->format, d, a, wide, sms, st); break;
        default: e = launch_read<float>(cache->format, d, a, wide, sms, st); break;
    }
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "read: %s", cudaGetErrorString(e));
}

}  // extern "C"
