// Attention of one new token per sequence over a paged key-value cache: the kernel.
//
// For each sequence and KV head the group's queries meet the same keys, so the cache is read
// once per KV head: 4 n_q d flops per 4 n_kv d bytes (bf16), far below what the tensor cores
// give per byte.  The kernel is bound by HBM; everything else has to stay out of its way.
//
// Work.  A unit is one page (16 keys) of one KV head and head tile.  All units of the batch,
// sequence after sequence, head after head, are cut into equal runs, one per block, however
// ragged the lengths are.  The warps of a block take its units in turn, each through a ring of
// its own in shared memory that cp.async fills ahead, across the ends of segments (a segment:
// the units of one sequence and head).  At a segment's end the block's warps join their
// states; a segment that spans blocks is joined by the block that finishes last.
//
// Softmax in base 2 with a running maximum m and sum l in fp32; O in fp32 accumulators.
//
// Products on mma.m16n8k16: S = Q K^T with 16 rows of queries, 8 keys and 16 elements of the
// head a step, O += P V with the same rows.  Neither operand of K or V is transposed or shuffled:
// * a lane's 16 bytes of a key row serve as its B fragments of several steps.  The order in
//   which a step's 16 elements stand for elements of the head is free as long as Q agrees;
// * the 16 keys of a unit are ordered so that the scores a lane gets are the ones its A
//   fragment of P needs, and V rows t, t + 4, t + 8, t + 12 give its B fragments by byte permutes.
//
// Precision.  K and V enter exactly: bf16 as stored; 8-bit codes as fp16, their scales applied
// to the scores and to the weights in fp32.  Q and P are carried as sums of 16-bit terms.  With
// at most 8 queries a group the second term's rows fill the upper half of the 16 (STACK), so two
// terms cost what one does; larger groups take 16 queries a tile and a pass per term.
//   bf16 cache: q and p as two terms (16 bits), or three where q or the result is fp32 (EXACT);
//   a bf16 q is one term exactly.
//   8-bit cache: two fp16 terms (22 bits).  q is scaled by a power of two per head, p by the
//   value's scale relative to the largest one so far, so that neither leaves fp16's range.
#pragma once
#include "ops.cuh"

namespace wici {

constexpr int kAttnWarps = 4;
constexpr int kAttnThreads = 32 * kAttnWarps;
constexpr int kAttnMaxBatch = 1024;   // sequences of a launch: their page counts are in shared memory
constexpr int kAttnPieceRows = 16;    // rows of a piece in the workspace (a head tile has 8 or 16)

struct AttnArg {
    HeadsArg q, out;
    CacheArg cache;
    const int32_t *pages, *lengths;
    float *lse;
    int32_t *status;
    int *tickets;                     // [blocks]: arrivals at the segment that starts in a block and leaves it
    float *pieces;                    // [blocks][2][kAttnPieceRows][D + 2]: O, m, l of a block's part of a segment
    int batch, q_heads, group, tiles; // head tiles of a KV head
    int max_pages, window;
    int q_dtype, out_dtype;
    bool q_wide, out_wide;
    float scale;
};

constexpr int attn_block(int fmt, int d) { return fmt == WICI_KV_BF16 ? kKvPage * d * 2 : kKvPage * (d + 4); }
constexpr size_t attn_piece_floats(int d) { return (size_t)kAttnPieceRows * (d + 2); }

template <int FMT, int D>
struct AttnShape {
    static constexpr int kBlock = attn_block(FMT, D);
    // ring slots of K and of V: what fits two blocks on an SM beside the join's buffer
    static constexpr int kKSlots = FMT == WICI_KV_BF16 && D == 128 ? 3 : 4;
    static constexpr int kVSlots = kKSlots - 1;
    static constexpr int kRing = (kKSlots + kVSlots) * kBlock;
    static constexpr int kJoinRow = D + 8;                         // floats: neighbouring rows in other banks
    static constexpr int kJoin = kAttnWarps * 8 * kJoinRow * 4;    // O of 8 rows of every warp
    static constexpr int kState = kAttnWarps * 8 * 2 * 4;          // m and l
    static constexpr int kSmem = kAttnWarps * kRing + kJoin + kState + (kAttnMaxBatch + 1) * 4 + 64;
};

// ------------------------------------------------------------------ PTX ----
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float lds32(uint32_t a) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
template <bool BF16>
__device__ __forceinline__ void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two fp32 values to 16 bits each (lo in the low half), and what the rounding left
template <bool BF16>
__device__ __forceinline__ uint32_t split2(float &lo, float &hi) {
    uint32_t w;
    if (BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        w = *(const uint32_t *)&h;
        lo -= __uint_as_float(w << 16);
        hi -= __uint_as_float(w & 0xFFFF0000u);
    } else {
        const __half2 h = __floats2half2_rn(lo, hi);
        w = *(const uint32_t *)&h;
        const float2 f = __half22float2(h);
        lo -= f.x;
        hi -= f.y;
    }
    return w;
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
        const __half2 p = decode2<FMT>(w), q = decode2<FMT>(w >> 16);
        lo = *(const uint32_t *)&p;
        hi = *(const uint32_t *)&q;
    }
}

// Where 16-byte chunk c of key row r stands in a ring slot.  The chunks of a row are permuted so
// that the 8 lanes of a shared-memory phase, which take rows i and i + 4 (K), or rows 0..3 and
// neighbouring chunks (V), meet 8 different bank groups.  Rows of 64 bytes share a line of 128 in pairs.
template <int ROW>
__device__ __forceinline__ int chunk_at(int r, int c) {
    if (ROW == 64) {
        const int line = r >> 1;
        return line * 128 + ((((r & 1) << 2 | c) ^ ((line & 1) << 1 ^ (line & 2) << 1)) << 4);
    }
    return r * ROW + ((c ^ ((r & 3) << 1) ^ ((r >> 2 & 1) * 5)) << 4);
}

__device__ __forceinline__ float load_any(const HeadsArg &t, int dtype, int64_t token, int head, int i) {
    switch (dtype) {
        case WICI_BF16: return to_f32(t.row<__nv_bfloat16>(token, head)[i]);
        case WICI_F16: return to_f32(t.row<__half>(token, head)[i]);
        default: return t.row<float>(token, head)[i];
    }
}
// 8 elements of q from element i on
__device__ __forceinline__ void load_q8(const AttnArg &a, int64_t token, int head, int i, float *v) {
    if (a.q_wide) {
        switch (a.q_dtype) {
            case WICI_BF16: load8<__nv_bfloat16, true>(a.q.row<__nv_bfloat16>(token, head) + i, 8, v); break;
            case WICI_F16: load8<__half, true>(a.q.row<__half>(token, head) + i, 8, v); break;
            default: load8<float, true>(a.q.row<float>(token, head) + i, 8, v); break;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = load_any(a.q, a.q_dtype, token, head, i + j);
    }
}
__device__ __forceinline__ void store_out4(const AttnArg &a, int64_t token, int head, int i, const float *v) {
    switch (a.out_dtype) {
        case WICI_F32: {
            float *p = a.out.row<float>(token, head) + i;
            if (a.out_wide) {
                *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
            } else {
                for (int j = 0; j < 4; ++j) p[j] = v[j];
            }
            break;
        }
        case WICI_F16: {
            __half *p = a.out.row<__half>(token, head) + i;
            alignas(8) __half e[4];
            for (int j = 0; j < 4; ++j) from_f32(v[j], e[j]);
            if (a.out_wide) {
                *(uint2 *)p = *(const uint2 *)e;
            } else {
                for (int j = 0; j < 4; ++j) p[j] = e[j];
            }
            break;
        }
        default: {
            __nv_bfloat16 *p = a.out.row<__nv_bfloat16>(token, head) + i;
            alignas(8) __nv_bfloat16 e[4];
            for (int j = 0; j < 4; ++j) from_f32(v[j], e[j]);
            if (a.out_wide) {
                *(uint2 *)p = *(const uint2 *)e;
            } else {
                for (int j = 0; j < 4; ++j) p[j] = e[j];
            }
        }
    }
}

// the keys of a sequence: [lo, n), none where the length is bad or not positive
struct Keys {
    int lo, n;
    bool bad;
    __device__ __forceinline__ int first_page() const { return lo / kKvPage; }
    __device__ __forceinline__ int page_count() const { return n > lo ? (n + kKvPage - 1) / kKvPage - lo / kKvPage : 0; }
};
__device__ __forceinline__ Keys keys_of(const AttnArg &a, int b) {
    Keys k;
    k.n = a.lengths[b];
    k.bad = k.n > a.max_pages * (int64_t)kKvPage;
    if (k.bad || k.n < 0) k.n = 0;
    k.lo = a.window && k.n > a.window ? k.n - a.window : 0;
    return k;
}

template <int FMT, int D, bool STACK, bool EXACT>
__global__ void __launch_bounds__(kAttnThreads, 2) paged_attention_kernel(const __grid_constant__ AttnArg a) {
    using S = AttnShape<FMT, D>;
    constexpr bool BF16 = FMT == WICI_KV_BF16;
    constexpr int ROW = BF16 ? 2 * D : D;                 // bytes of a key row
    constexpr int CHUNKS = ROW / 16;
    constexpr int PER = BF16 ? 8 : 16;                    // elements of a chunk
    constexpr int HT = STACK ? 8 : 16;                    // queries of a head tile
    constexpr int R = STACK ? 1 : 2;                      // queries whose rows a lane holds
    constexpr int TQ = BF16 && EXACT ? 3 : STACK || !BF16 ? 2 : 1;
    constexpr int TP = BF16 && EXACT ? 3 : 2;
    constexpr int QPASS = STACK ? (TQ + 1) / 2 : TQ, PPASS = STACK ? (TP + 1) / 2 : TP;
    constexpr int STEPS = D / 16, NT = D / 8;
    constexpr int KS = S::kKSlots, VS = S::kVSlots;
    constexpr float kPUnit = BF16 ? 1.f : 4096.f;         // what weights are scaled up by (fp16: far from its smallest)

    extern __shared__ __align__(128) uint8_t smem[];
    float *join = (float *)(smem + kAttnWarps * S::kRing);            // [warp][8][kJoinRow]
    float2 *state = (float2 *)((uint8_t *)join + S::kJoin);           // [warp][8]: m, l
    int *prefix = (int *)((uint8_t *)state + S::kState);              // [batch + 1]: pages of the sequences before
    int *sflag = prefix + kAttnMaxBatch + 1;                          // [8]

    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * S::kRing;
    griddep_wait();

    // ---- page counts of all sequences, and their sums ----
    {
        const int per = (a.batch + kAttnThreads - 1) / kAttnThreads;
        const int b0 = min(a.batch, (int)threadIdx.x * per), b1 = min(a.batch, b0 + per);
        int sum = 0;
        for (int b = b0; b < b1; ++b) sum += keys_of(a, b).page_count();
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) sflag[warp] = incl;
        __syncthreads();
        int at = incl - sum;
        for (int w = 0; w < warp; ++w) at += sflag[w];
        for (int b = b0; b < b1; ++b) {
            prefix[b] = at;
            at += keys_of(a, b).page_count();
        }
        if (b1 == a.batch) prefix[a.batch] = at;
        __syncthreads();
    }
    const int HH = a.cache.kv_heads * a.tiles;
    const int64_t U = (int64_t)prefix[a.batch] * HH;

    // sequences without keys: zeros, or NaN where the length is bad
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
        if (prefix[b + 1] != prefix[b]) continue;
        const bool bad = keys_of(a, b).bad;
        const float fill = bad ? __uint_as_float(0x7FC00000u) : 0.f, f4[4] = {fill, fill, fill, fill};
        for (int i = threadIdx.x; i < a.q_heads * (D / 4); i += kAttnThreads)
            store_out4(a, b, i / (D / 4), i % (D / 4) * 4, f4);
        if (a.lse)
            for (int h = threadIdx.x; h < a.q_heads; h += kAttnThreads)
                a.lse[(int64_t)b * a.q_heads + h] = bad ? fill : -INFINITY;
        if (bad && threadIdx.x == 0 && a.status) atomicOr(a.status, WICI_BAD_LENGTH);
    }

    // ---- this block's run of units ----
    const int64_t blocks = min((int64_t)gridDim.x, (U + 15) / 16);    // at least 16 units a block
    if (blockIdx.x >= blocks) return;
    const int64_t u0 = blockIdx.x * U / blocks, u1 = (blockIdx.x + 1) * U / blocks;
    const int count = (int)(u1 - u0);
    const int mine = count > warp ? (count - warp + kAttnWarps - 1) / kAttnWarps : 0;   // units of this warp

    auto sequence_of = [&](int q) {       // the last b with prefix[b] <= q: it has pages
        int lo = 0, hi = a.batch;         // prefix[lo] <= q < prefix[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (prefix[mid] <= q) lo = mid; else hi = mid;
        }
        return lo;
    };

    // ---- issue side: lane l knows unit 32 k + l of this warp's ----
    struct Desc {
        int page;      // -1: bad
        int info;      // kv head | first valid row << 16 | rows end << 24
    };
    auto describe = [&](int i) {
        Desc d = {-1, 0};
        if (i >= mine) return d;
        const int64_t u = u0 + warp + (int64_t)kAttnWarps * i;
        const int b = sequence_of((int)(u / HH));
        const int n_b = prefix[b + 1] - prefix[b];
        const int64_t r = u - (int64_t)prefix[b] * HH;
        const int head = (int)(r / n_b), p = (int)(r - (int64_t)head * n_b);
        const Keys k = keys_of(a, b);
        const int at = k.first_page() + p;
        d.page = a.pages[(int64_t)b * a.max_pages + at];
        if (d.page < 0 || d.page >= a.cache.n_pages) d.page = -1;
        const int first = max(0, k.lo - at * kKvPage), end = min(kKvPage, k.n - at * kKvPage);
        d.info = head / a.tiles | first << 16 | end << 24;
        return d;
    };
    Desc cur = describe(lane), next = describe(32 + lane);
    int issued = 0;                       // K's of units issued; V's follow one behind
    uint32_t bad_units = 0;               // bit i % 32: unit i has a bad page
    int last_page = -1, last_info = 0;

    auto copy_block = [&](uint32_t dst, int page, int info, bool v) {
        const int first = info >> 16 & 255, end = info >> 24;
        const uint8_t *src = a.cache.data + page * a.cache.page_stride +
                             (int64_t)((info & 0xFFFF) + (v ? a.cache.kv_heads : 0)) * S::kBlock;
#pragma unroll
        for (int i = 0; i < kKvPage * CHUNKS / 32; ++i) {
            const int c = i * 32 + lane, r = c / CHUNKS, x = c % CHUNKS;
            // rows without a key of the sequence are zeroed: what the cache holds there is anything
            cp_async16(dst + chunk_at<ROW>(r, x), src + c * 16, r >= first && r < end ? 16 : 0);
        }
        if (!BF16 && lane < 4) cp_async16(dst + kKvPage * D + lane * 16, src + kKvPage * D + lane * 16, 16);
    };
    // group j: K of unit j and V of the one before it (none past the last unit: the groups still count)
    auto issue = [&]() {
        if (issued && (issued & 31) == 0) {
            cur = next;
            next = describe(issued + 32 + lane);
        }
        const int page = __shfl_sync(0xffffffffu, cur.page, issued & 31);
        const int info = __shfl_sync(0xffffffffu, cur.info, issued & 31);
        if (issued < mine) {
            if (page < 0) {
                bad_units |= 1u << (issued & 31);
                if (lane == 0 && a.status) atomicOr(a.status, WICI_BAD_PAGE);
            } else {
                copy_block(ring + issued % KS * S::kBlock, page, info, false);
            }
        }
        if (last_page >= 0)
            copy_block(ring + KS * S::kBlock + (issued - 1) % VS * S::kBlock, last_page, last_info, true);
        last_page = issued < mine ? page : -1;
        last_info = info;
        ++issued;
        cp_commit();
    };
    for (int i = 0; i < KS; ++i) issue();

    // ---- segments ----
    int seg_b = sequence_of((int)(u0 / HH));
    int seg_head;
    int64_t seg_start;                    // first unit
    {
        const int n_b = prefix[seg_b + 1] - prefix[seg_b];
        const int64_t r = u0 - (int64_t)prefix[seg_b] * HH;
        seg_head = (int)(r / n_b);
        seg_start = u0 - (r - (int64_t)seg_head * n_b);
    }
    int done = 0;                         // units of this warp computed
    for (int64_t u = u0; u < u1;) {
        const int n_b = prefix[seg_b + 1] - prefix[seg_b];
        const int64_t seg_end = seg_start + n_b, stop = min(seg_end, u1);
        const Keys keys = keys_of(a, seg_b);
        const int kvh = seg_head / a.tiles, row0 = seg_head % a.tiles * HT;   // first query of the tile in the group
        const int rows = min(HT, a.group - row0);
        const int head0 = kvh * a.group + row0;

        // ---- Q fragments: step s of a chunk takes 4 of its elements ----
        uint32_t qf[QPASS][STEPS][4];
        float cq[R];                      // scores to base-2 logits
        const bool any = done < mine && u0 + warp + (int64_t)kAttnWarps * done < stop;
#pragma unroll
        for (int r = 0; r < R; ++r) cq[r] = a.scale * 1.44269504088896340736f;
        if (any) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int row = g + 8 * r;
                float x[STEPS][4];
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < STEPS / 2; ++i) {
                    float v[8];
                    // bf16: chunk 4 i + t; 8-bit: half i % 2 of chunk 4 (i / 2) + t
                    const int e0 = BF16 ? 8 * (4 * i + t) : 16 * (4 * (i / 2) + t) + 8 * (i % 2);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = 0.f;
                    if (row < rows) load_q8(a, seg_b, head0 + row, e0, v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[2 * i + j / 4][j % 4] = v[j];
                        top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
                    }
                }
                if (!BF16) {
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    // 2^(13 - exponent): the largest magnitude to [2^13, 2^14)
                    int e = (int)(top >> 23) - 127 - 13;
                    e = top >= kInfBits || top == 0 ? 0 : max(-126, min(126, e));
                    const float down = __int_as_float((127 - e) << 23);
                    cq[r] *= __int_as_float((127 + e) << 23);
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[s][j] *= down;
                }
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
#pragma unroll
                    for (int k = 0; k < QPASS; ++k) {
                        if (STACK) {
                            qf[k][s][0] = split2<BF16>(x[s][0], x[s][1]);
                            qf[k][s][2] = split2<BF16>(x[s][2], x[s][3]);
                            qf[k][s][1] = 2 * k + 1 < TQ ? split2<BF16>(x[s][0], x[s][1]) : 0u;
                            qf[k][s][3] = 2 * k + 1 < TQ ? split2<BF16>(x[s][2], x[s][3]) : 0u;
                        } else {
                            qf[k][s][r] = split2<BF16>(x[s][0], x[s][1]);
                            qf[k][s][2 + r] = split2<BF16>(x[s][2], x[s][3]);
                        }
                    }
                }
            }
        }

        float m[R], l[R], o[NT][4];
#pragma unroll
        for (int r = 0; r < R; ++r) m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][j] = 0.f;
        float vref = 0x1p-125f, vinv = 0x1p125f;      // 8-bit: a power of two, at least a quarter of the largest V scale

        // ---- units of this segment ----
        for (; done < mine; ++done) {
            const int64_t unit = u0 + warp + (int64_t)kAttnWarps * done;
            if (unit >= stop) break;
            // group `done` brings K; the KS - 1 after it may be on their way
            cp_wait<KS - 1>();
            __syncwarp();
            const int base_key = (keys.first_page() + (int)(unit - seg_start)) * kKvPage;
            const uint32_t ks = ring + done % KS * S::kBlock, vs = ring + KS * S::kBlock + done % VS * S::kBlock;

            float c[2][2][4];                                // [8 keys][even, odd steps]
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < 4; ++j) c[n][e][j] = 0.f;
#pragma unroll
            for (int i = 0; i < CHUNKS / 4; ++i) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int r = (g >> 1) + (g & 1) * 4 + 8 * n;   // the key of column g
                    const uint4 w = lds128(ks + chunk_at<ROW>(r, 4 * i + t));
                    if (BF16) {
#pragma unroll
                        for (int k = 0; k < QPASS; ++k) {
                            mma16816<true>(c[n][0], qf[k][2 * i], w.x, w.y);
                            mma16816<true>(c[n][1], qf[k][2 * i + 1], w.z, w.w);
                        }
                    } else {
                        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            uint32_t b0, b1;
                            decode4<FMT>(word[s], b0, b1);
#pragma unroll
                            for (int k = 0; k < QPASS; ++k) mma16816<false>(c[n][s & 1], qf[k][4 * i + s], b0, b1);
                        }
                    }
                }
            }
            // x[r][j]: query g + 8 r, key t + 4 j
            float x[R][4], vscale[4];
            float vtop = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = j >> 1, col = j & 1, key = t + 4 * j;
                const bool valid = base_key + key >= keys.lo && base_key + key < keys.n;
                float ksc = 1.f;
                if (!BF16) ksc = lds32(ks + kKvPage * D + key * 4);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float a0 = c[n][0][col + 2 * r] + c[n][1][col + 2 * r];
                    const float dot = STACK ? a0 + (c[n][0][col + 2] + c[n][1][col + 2]) : a0;
                    x[r][j] = valid ? dot * ksc * cq[r] : -INFINITY;
                }
            }
            float up[R];
            bool grew = false;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float top = fmaxf(fmaxf(x[r][0], x[r][1]), fmaxf(x[r][2], x[r][3]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                up[r] = fmaxf(m[r], top);
                grew |= up[r] > m[r];
            }
            // V of this unit is in the next group
            cp_wait<KS - 2>();
            __syncwarp();
            float ratio = 1.f;
            if (!BF16) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = t + 4 * j;
                    const bool valid = base_key + key >= keys.lo && base_key + key < keys.n;
                    vscale[j] = valid ? lds32(vs + kKvPage * D + key * 4) : 0.f;
                    vtop = fmaxf(vtop, vscale[j]);
                }
                vtop = fmaxf(vtop, __shfl_xor_sync(0xffffffffu, vtop, 1));
                vtop = fmaxf(vtop, __shfl_xor_sync(0xffffffffu, vtop, 2));
                if (vtop > vref) {                           // the same in every lane
                    const uint32_t e = min((__float_as_uint(vtop) + 0x7FFFFFu) & 0x7F800000u, 0x7E800000u);
                    const float ref = __uint_as_float(e);
                    ratio = vref * __uint_as_float(0x7F000000u - e);
                    vref = ref;
                    vinv = __uint_as_float(0x7F000000u - e);
                    grew = true;
                }
            }
            if (__any_sync(0xffffffffu, grew)) {
                float f[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    f[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - up[r]);   // nothing yet: zeros
                    l[r] *= f[r];
                    f[r] *= ratio;
                    m[r] = up[r];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    o[n][0] *= f[0];
                    o[n][1] *= f[0];
                    o[n][2] *= f[R - 1];
                    o[n][3] *= f[R - 1];
                }
            }
            uint32_t pf[PPASS][4];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float ref = m[r] == -INFINITY ? 0.f : m[r];
                float p[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    p[j] = ex2(x[r][j] - ref);
                    l[r] += p[j];
                    if (!BF16) p[j] *= vscale[j] * vinv * kPUnit;
                }
#pragma unroll
                for (int k = 0; k < PPASS; ++k) {
                    if (STACK) {
                        pf[k][0] = split2<BF16>(p[0], p[1]);
                        pf[k][2] = split2<BF16>(p[2], p[3]);
                        pf[k][1] = 2 * k + 1 < TP ? split2<BF16>(p[0], p[1]) : 0u;
                        pf[k][3] = 2 * k + 1 < TP ? split2<BF16>(p[2], p[3]) : 0u;
                    } else {
                        pf[k][r] = split2<BF16>(p[0], p[1]);
                        pf[k][2 + r] = split2<BF16>(p[2], p[3]);
                    }
                }
            }
            // V: rows t + 4 i; column g of tile n is element PER * (g + 8 jj) + e of the head (n = PER jj + e),
            // or 8 g + n where a lane takes half a chunk (8-bit, d 64)
            if (BF16) {
#pragma unroll
                for (int jj = 0; jj < CHUNKS / 8; ++jj) {
                    uint32_t w[4][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint4 q = lds128(vs + chunk_at<ROW>(t + 4 * i, g + 8 * jj));
                        w[i][0] = q.x, w[i][1] = q.y, w[i][2] = q.z, w[i][3] = q.w;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t sel = e & 1 ? 0x7632 : 0x5410;
                        const uint32_t b0 = __byte_perm(w[0][e / 2], w[1][e / 2], sel);
                        const uint32_t b1 = __byte_perm(w[2][e / 2], w[3][e / 2], sel);
#pragma unroll
                        for (int k = 0; k < PPASS; ++k) mma16816<true>(o[8 * jj + e], pf[k], b0, b1);
                    }
                }
            } else {
                constexpr int WORDS = D / 32;              // 4-byte words of a row that a lane takes
                uint32_t w[4][WORDS];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (D == 128) {
                        const uint4 q = lds128(vs + chunk_at<ROW>(t + 4 * i, g));
                        w[i][0] = q.x, w[i][1] = q.y, w[i][WORDS - 2] = q.z, w[i][WORDS - 1] = q.w;
                    } else {
                        const uint2 q = lds64(vs + chunk_at<ROW>(t + 4 * i, g >> 1) + (g & 1) * 8);
                        w[i][0] = q.x, w[i][1] = q.y;
                    }
                }
#pragma unroll
                for (int x4 = 0; x4 < WORDS; ++x4) {
                    uint32_t h[4][2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) decode4<FMT>(w[i][x4], h[i][0], h[i][1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t sel = e & 1 ? 0x7632 : 0x5410;
                        const uint32_t b0 = __byte_perm(h[0][e / 2], h[1][e / 2], sel);
                        const uint32_t b1 = __byte_perm(h[2][e / 2], h[3][e / 2], sel);
#pragma unroll
                        for (int k = 0; k < PPASS; ++k) mma16816<false>(o[4 * x4 + e], pf[k], b0, b1);
                    }
                }
            }
            if (bad_units >> (done & 31) & 1) {
                bad_units &= ~(1u << (done & 31));
#pragma unroll
                for (int r = 0; r < R; ++r) l[r] = __uint_as_float(0x7FC00000u);
            }
            __syncwarp();                                   // every lane has read the slots
            issue();
        }

        // ---- join the block's warps, 8 rows at a time ----
#pragma unroll
        for (int r = 0; r < R; ++r) {
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        }
        const bool whole = seg_start >= u0 && seg_end <= u1;
        float *piece = a.pieces + ((int64_t)blockIdx.x * 2 + (seg_start >= u0 ? 1 : 0)) * attn_piece_floats(D);
        const float unit_of_o = BF16 ? 1.f : vref / kPUnit;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            __syncthreads();                                // the buffer's last readers are done
            float *mine_o = join + (warp * 8 + g) * S::kJoinRow;
#pragma unroll
            for (int n = 0; n < NT; n += 4) {
                // columns 2 t and 2 t + 1 of tiles n .. n + 3: four adjacent elements each
                constexpr int per = BF16 || D == 64 ? 8 : 16;
                float v[2][4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        v[c][i] = (STACK ? o[n + i][c] + o[n + i][c + 2] : o[n + i][2 * r + c]) * unit_of_o;
                float *dst = mine_o + per * (2 * t + 8 * (n / per)) + n % per;
                *(float4 *)dst = make_float4(v[0][0], v[0][1], v[0][2], v[0][3]);
                *(float4 *)(dst + per) = make_float4(v[1][0], v[1][1], v[1][2], v[1][3]);
            }
            if (t == 0) state[warp * 8 + g] = make_float2(m[r], l[r]);
            __syncthreads();
            for (int i = threadIdx.x; i < 8 * (D / 4); i += kAttnThreads) {
                const int row = i / (D / 4), d0 = i % (D / 4) * 4;
                if (row + 8 * r >= rows) continue;
                float top = -INFINITY, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kAttnWarps; ++w) top = fmaxf(top, state[w * 8 + row].x);
#pragma unroll
                for (int w = 0; w < kAttnWarps; ++w) {
                    const float2 s = state[w * 8 + row];
                    const float f = s.x == -INFINITY ? 0.f : ex2(s.x - top);
                    sum += s.y * f;
                    const float4 q = *(const float4 *)(join + (w * 8 + row) * S::kJoinRow + d0);
                    v[0] += q.x * f, v[1] += q.y * f, v[2] += q.z * f, v[3] += q.w * f;
                }
                if (whole) {
                    const float inv = 1.f / sum;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] *= inv;
                    store_out4(a, seg_b, head0 + row + 8 * r, d0, v);
                    if (d0 == 0 && a.lse)
                        a.lse[(int64_t)seg_b * a.q_heads + head0 + row + 8 * r] =
                            (top + log2f(sum)) * 0.693147180559945309417f;
                } else {
                    float *dst = piece + (row + 8 * r) * D + d0;
                    *(float4 *)dst = make_float4(v[0], v[1], v[2], v[3]);
                    if (d0 == 0) {
                        float2 *ml = (float2 *)(piece + kAttnPieceRows * D) + row + 8 * r;
                        *ml = make_float2(top, sum);
                    }
                }
            }
        }
        if (!whole) {
            // blocks i0 .. i1 hold the segment; the one that arrives last joins their pieces in order
            const int i0 = (int)(((seg_start + 1) * blocks - 1) / U), i1 = (int)((seg_end * blocks - 1) / U);
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                const int n = atomicAdd(a.tickets + i0, 1);
                sflag[0] = n == i1 - i0;
                if (n == i1 - i0) a.tickets[i0] = 0;
            }
            __syncthreads();
            if (sflag[0]) {
                __threadfence();
                for (int i = threadIdx.x; i < rows * (D / 4); i += kAttnThreads) {
                    const int row = i / (D / 4), d0 = i % (D / 4) * 4;
                    float top = -INFINITY, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
                    for (int p = i0; p <= i1; ++p) {
                        const float *src = a.pieces + ((int64_t)p * 2 + (p == i0)) * attn_piece_floats(D);
                        const float2 s = __ldcg((const float2 *)(src + kAttnPieceRows * D) + row);
                        const float4 q = __ldcg((const float4 *)(src + row * D + d0));
                        const float up = fmaxf(top, s.x), ref = up == -INFINITY ? 0.f : up;
                        const float fo = ex2(top - ref), fn = ex2(s.x - ref);
                        sum = sum * fo + s.y * fn;
                        v[0] = v[0] * fo + q.x * fn, v[1] = v[1] * fo + q.y * fn;
                        v[2] = v[2] * fo + q.z * fn, v[3] = v[3] * fo + q.w * fn;
                        top = up;
                    }
                    const float inv = 1.f / sum;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] *= inv;
                    store_out4(a, seg_b, head0 + row, d0, v);
                    if (d0 == 0 && a.lse)
                        a.lse[(int64_t)seg_b * a.q_heads + head0 + row] = (top + log2f(sum)) * 0.693147180559945309417f;
                }
            }
            __syncthreads();                                // sflag is free again
        }

        // ---- the next segment ----
        u = stop;
        if (u < u1) {
            seg_start = seg_end;
            if (++seg_head == HH) {
                seg_head = 0;
                do ++seg_b; while (prefix[seg_b + 1] == prefix[seg_b]);
            }
        }
    }
    cp_wait<0>();
}

// Launches, and kernel limits of the current device; one translation unit per format.
cudaError_t launch_attention_bf16(int d, const AttnArg &a, bool stack, bool exact, int grid, cudaStream_t st);
cudaError_t launch_attention_int8(int d, const AttnArg &a, bool stack, int grid, cudaStream_t st);
cudaError_t launch_attention_e4m3(int d, const AttnArg &a, bool stack, int grid, cudaStream_t st);
cudaError_t setup_attention_bf16();
cudaError_t setup_attention_int8();
cudaError_t setup_attention_e4m3();

template <int FMT, int D, bool STACK, bool EXACT>
cudaError_t launch_attention(const AttnArg &a, int grid, cudaStream_t st) {
    return launch_kernel(paged_attention_kernel<FMT, D, STACK, EXACT>, dim3(grid), kAttnThreads,
                         AttnShape<FMT, D>::kSmem, st, 1, true, a);
}
template <int FMT, int D, bool STACK, bool EXACT>
cudaError_t limit_attention() {
    return cudaFuncSetAttribute(paged_attention_kernel<FMT, D, STACK, EXACT>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, AttnShape<FMT, D>::kSmem);
}

}  // namespace wici
