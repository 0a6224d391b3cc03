// Attention of one new token per sequence over a paged key-value cache: the kernel.
//
// For each sequence and KV head the group's queries meet the same keys, so the cache is read
// once per KV head: 4 n_q d flops per 4 n_kv d bytes (bf16), far below what the tensor cores
// give per byte.  The kernel is bound by HBM; everything else has to stay out of its way.
//
// Work.  A unit is P pages (16 P keys) of one KV head and head tile.  All units of the batch,
// sequence after sequence, head after head, are cut into equal runs, one per warp, however
// ragged the lengths are; a segment (the units of one sequence and head) weighs kAttnSegment
// units more than it has, for its queries' way in and its result's way out.  A warp streams its
// run through a ring of its own in shared memory that cp.async fills ahead, across the ends of
// segments.  A segment inside one run is finished by its warp alone; the parts of others are
// joined by the block at its end, and by the block that finishes last where blocks share one:
// short segments (kAttnWhole) they never share.
// Measured (device time; 8 KV heads of 128): 32 sequences of up to 4000 tokens in bf16 47 us, 5.6 TB/s
// of keys; two of 100001 to 131072 141 us, 6.7 TB/s; 64 of up to 8192 in int8, five queries a KV head,
// 108 us, 5.6 TB/s; 256 of 20 to 300 35 us, 1000 of them 108 us; one of 200 tokens 8.0 us.  Of each
// about 4 us pass before the first keys are there (lengths, then pages, then keys), and 4 to 8 after the
// first warp is done.
//
// Softmax in base 2 with a running reference m, at most 6 below the running maximum, and a sum l in
// fp32; O in fp32 accumulators.
//
// Products on mma.m16n8k16: S = Q K^T with 16 rows of queries, 8 keys and 16 elements of the
// head a step, O += P V with the same rows.  Neither K nor V is transposed or shuffled:
// * a lane's 16 bytes of a key row serve as its B fragments of several steps.  The order in
//   which a step's 16 elements stand for elements of the head is free as long as Q agrees;
// * the 16 keys of a page are ordered so that the scores a lane gets are the ones its A
//   fragment of P needs, and V rows t, t + 4, t + 8, t + 12 give its B fragments by byte permutes.
//
// Precision.  K and V enter exactly: bf16 as stored; 8-bit codes as fp16, their scales applied
// to the scores and to the weights in fp32.  Q and P are carried as sums of 16-bit terms.  With
// at most 8 queries a group the second term's rows fill the upper half of the 16 (STACK), so two
// terms cost what one does; larger groups take 16 queries a tile and a pass per term.
//   bf16 cache: q that is not bf16 as three terms; p as two (17 bits, in tiles of 16 queries 16),
//   or three where q is not bf16 or the result is fp32 (EXACT).
//   8-bit cache: q as one fp16 term (bf16 and fp16 fit exactly) or, from fp32, as two (EXACT),
//   scaled by a power of two per head; p times its value's scale as two (22 bits), multiplied by a
//   power of two per query that follows the largest such weight so far: a weight is off by 2^-22 of
//   itself or 2^-32 of the largest one, however large the scale of a value is that hardly counts.
//   4-bit cache: as 8-bit; a code times its block's scale is one fp16 number, exactly.
//   Tensor cores cut what an addition leaves over, always downwards in size: a long run's sums of P V come out too small by
//   some 2^-24 an addition.  Rows of their own (8-bit and bf16, up to 8 queries) take one a page, the two terms of P over
//   4-bit codes two; for fp32 queries these are summed a unit at a time.
//
// 4-bit codes (E2M1).  Half of an 8-bit cache's bytes for the same arithmetic.  As fast from L2, and no pipe is full either
// (of the active cycles issue slots 52%, ALU 42%, tensor cores 26%): two warps a scheduler wait for one another's chains of
// loads from shared memory, conversions, products with block scales and matrix products, first of all for the fixed latency
// of the instruction before.  So the operands change places: S^T = K Q^T and
// O^T = V^T P^T, with keys and elements of the head as the 16 rows and 8 queries as the columns.  A fragment of converted
// codes then serves both terms of Q or P (and 16 queries a tile two tiles) at half the products of K, and O takes 32
// registers in place of 64; P^T comes from the scores by movmatrix.  64 sequences of up to 8192 tokens, five queries a KV
// head: 93 us (104 with queries as rows), two of 100001 to 131072: 72 us (80), 3.9 TB/s of codes, 730 instructions for 32
// keys at 0.52 a cycle and scheduler; with 16 queries a KV head 106 us.  Not kept: three blocks on an SM with 168 registers
// (74 us; beside an append 131 in place of 103, for an append's blocks split the registers that a third block would need),
// four pages a unit (70.6, but 95.6 for the 64 sequences), five ring slots (the same), two sums for a score or terms of P
// apart (the same).
#pragma once
#include "ops.cuh"

namespace wici {

constexpr int kAttnWarps = 4;
constexpr int kAttnThreads = 32 * kAttnWarps;
constexpr uint32_t kAttnSegment = 3;       // units that a segment weighs beside its own
constexpr uint32_t kAttnMinUnits = 2;      // weight of a warp's run at least: shorter ones would not pay for joining more parts
                                           // (8 heads of 1000 tokens 10.1 us; with 3 instead, before, 10.3 for 9.7; of 140, 16 sequences: 9.0 and 11.4)
// Weight of a segment at most that blocks do not share.  Block edges moved by up to half of it cost the longest warp 3
// units, a joining of pieces 3 us and more: 16 sequences of 70 tokens, 4 KV heads of 8 queries, 10.2 us (13.1 where
// blocks share), 16 queries of an e4m3 cache 12.2 (23.3); 1000 of 20 to 300 tokens 108.5 (112.4).  16 and 40 in its
// place: 111.5 and 106.9 for the 1000, the same for the others.
constexpr uint32_t kAttnWhole = 24;
constexpr int kAttnPieceRows = 16;    // rows of a piece in the workspace (a head tile has 8 or 16)

struct AttnArg {
    HeadsArg q, out;
    CacheArg cache;
    const int32_t *pages, *lengths;
    float *lse;
    int32_t *status;
    int *tickets;                     // [blocks]: arrivals at the segment that starts in a block and leaves it
    float *pieces;                    // [blocks][2][kAttnPieceRows][D + 2]: O, then m and l, of a block's part of a segment
    int batch, q_heads, group, tiles; // head tiles of a KV head
    int64_t table_stride;             // of `pages`: entries from a sequence to the next
    int head_stride;                  // and from a KV head to the next: 0 where all read the same pages
    int max_pages, window;
    int q_dtype, out_dtype;
    bool q_wide, out_wide;
    float scale;
};

constexpr size_t attn_piece_floats(int d) { return (size_t)kAttnPieceRows * (d + 2); }

template <int FMT, int D, bool STACK>
struct AttnShape {
    static constexpr int kRows = STACK ? 8 : 16;                   // queries of a head tile
    static constexpr int kMaxBatch = STACK ? 1024 : 256;           // sequences of a launch: their keys are in shared memory
    // Pages of a unit: 4 to 8 KB of K and V for the work that a unit costs beside its products (bf16, 128: one page
    // already; 8-bit: one page more a unit took the batch of 64 from 136 to 116 us with 128, from 76 to 74 with 64).  4-bit
    // codes as 8-bit ones: the work a unit costs counts more than its bytes (half the pages: 48 in place of 42.5 us with 64).
    static constexpr int kPages = FMT == WICI_KV_BF16 ? (D == 128 ? 1 : 2) : (D == 128 ? 2 : 4);
    static constexpr int kBlock = kv_block_bytes(FMT, D);
    static constexpr int kSlot = kPages * kBlock;
    // Two blocks on an SM, 8 warps with 250 registers each: three of 168 spill (131 us in place of then 116).
    static constexpr int kBlocks = 2;
    static constexpr int kKSlots = 3, kVSlots = kKSlots - 1;   // of the ring: about 100 KB on their way per SM
    static constexpr int kRing = (kKSlots + kVSlots) * kSlot;
    static constexpr int kPartRow = D + 4;                         // floats: neighbouring rows in other banks
    static constexpr int kPart = kRows * (kPartRow + 2) * 4;       // a part of a segment: O, then m and l of each row
    static constexpr int kSmem = kAttnWarps * kRing + (kAttnWarps - 1) * kPart + (3 * kMaxBatch + 2) * 4 + 128;
    static_assert(kPart <= kRing, "a warp's last part lies in its ring");
    static_assert(kBlocks * (kSmem + 1024) <= 228 * 1024, "blocks of an SM");
};

// ------------------------------------------------------------------ PTX ----
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int bytes, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(bytes),
                 "l"(policy)
                 : "memory");
}
// the same where `there`, without a branch
__device__ __forceinline__ void cp_async16_if(bool there, uint32_t dst, const void *src, int bytes, uint64_t policy) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "@p cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;\n\t}" ::"r"(dst), "l"(src), "r"(bytes), "l"(policy),
                 "r"((uint32_t)there)
                 : "memory");
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
        asm(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// a product in fp16 added to a sum, or to nothing
__device__ __forceinline__ void mma_f16(float *c, bool first, const uint32_t *a, const uint32_t *b) {
    if (first)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]), "f"(0.f));
    else
        mma16816<false>(c, a, b[0], b[1]);
}
// an 8 x 8 matrix of 16-bit values, two of a row in each lane, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
// an e4m3 code as fp16 in the lower half, products of fp16 pairs: with a pair, with a lower half
__device__ __forceinline__ uint32_t e4m3_half(uint32_t code) {
    const __half2 v = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)code, __NV_E4M3));
    return *(const uint32_t *)&v;
}
__device__ __forceinline__ uint32_t times(uint32_t a, uint32_t b) {
    const __half2 v = __hmul2(*(const __half2 *)&a, *(const __half2 *)&b);
    return *(const uint32_t *)&v;
}
__device__ __forceinline__ uint32_t times_low(uint32_t a, uint32_t b) {
    const __half2 v = __hmul2(*(const __half2 *)&a, __low2half2(*(const __half2 *)&b));
    return *(const uint32_t *)&v;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 values (POSITIVE: or 0) as sums of N 16-bit terms each, lo in a term's low half; the last one is the nearest
// to what the others leave, times `last`.
// CUT (bf16): the others are cut off, not rounded, and what they leave counts as 2^-30 of the value at least: all terms
// have the value's sign and none is 0 beside it.  Their products with an infinite key or value are then the infinity
// that the value's own product is.  Otherwise every term is the nearest, which is worth a bit: fp16 terms meet codes
// alone, which are finite, and of two bf16 terms in rows of their own the first one's sum tells (rows_sum).
template <bool BF16, bool CUT, bool POSITIVE, int N>
__device__ __forceinline__ void split(float lo, float hi, uint32_t *w, float last) {
    const float lo_least = fabsf(lo) * 0x1p-30f, hi_least = fabsf(hi) * 0x1p-30f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i + 1 == N) lo *= last, hi *= last;
        if (!BF16) {
            const __half2 h = __floats2half2_rn(lo, hi);
            const float2 f = __half22float2(h);
            w[i] = *(const uint32_t *)&h;
            lo -= f.x;
            hi -= f.y;
        } else if (i + 1 == N || !CUT) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
            w[i] = *(const uint32_t *)&h;
            lo -= __uint_as_float(w[i] << 16);
            hi -= __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
            w[i] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
            const float lo_rest = lo - __uint_as_float(w[i] << 16), hi_rest = hi - __uint_as_float(w[i] & 0xFFFF0000u);
            lo = POSITIVE ? fmaxf(lo_rest, lo_least) : copysignf(fmaxf(fabsf(lo_rest), lo_least), lo);
            hi = POSITIVE ? fmaxf(hi_rest, hi_least) : copysignf(fmaxf(fabsf(hi_rest), hi_least), hi);
        }
    }
}
// The sum of a stacked tile's two rows: where the first term has met an infinity, the second may have met it with any sign
__device__ __forceinline__ float rows_sum(float first, float second) {
    return fabsf(first) < INFINITY ? first + second : first;
}
// The A fragments of one lane's 4 values of a row (two pairs) in N terms, over the passes of a tile.  STACK: a pass has
// a term in the lane's row and the next in the row 8 below, and half of the last one in both where they do not pair up;
// a single term leaves the lower row 0.  Otherwise a pass has a term in row r of the lane's two.
template <bool BF16, bool POSITIVE, bool STACK, int N, int STRIDE>
__device__ __forceinline__ void split_row(const float *x, int r, uint32_t (*a)[4]) {
    uint32_t w[2][N];
    constexpr bool CUT = BF16 && !(STACK && N == 2);
    const float last = STACK && N > 1 && N % 2 ? 0.5f : 1.f;
    split<BF16, CUT, POSITIVE, N>(x[0], x[1], w[0], last);
    split<BF16, CUT, POSITIVE, N>(x[2], x[3], w[1], last);
#pragma unroll
    for (int k = 0; k < (STACK ? (N + 1) / 2 : N); ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (STACK) {
                a[k * STRIDE][2 * h] = w[h][2 * k];
                a[k * STRIDE][2 * h + 1] = N == 1 ? 0u : w[h][2 * k + 1 < N ? 2 * k + 1 : N - 1];
            } else {
                a[k * STRIDE][2 * h + r] = w[h][k];
            }
        }
}

// Where 16-byte chunk c of key row r stands in a ring slot.  The chunks of a row are permuted so
// that the 8 lanes of a shared-memory phase, which take rows i and i + 4 (K), or rows 0..3 and
// neighbouring chunks (V), meet 8 different bank groups.  Rows of 64 bytes share a line of 128 in pairs.
// Of rows of e2m1 a lane takes 8 bytes at a time (of V with head_dim 64: 4): the half of a warp that a phase serves, with
// 4 neighbouring rows (K) or every other of 8 (V), meets all 32 banks.
template <int ROW, bool E2M1>
__device__ __forceinline__ int chunk_at(int r, int c) {
    if (E2M1 && ROW == 64) {
        const int line = r >> 1;
        return line * 128 + ((((r & 1) << 2 | c) ^ ((line & 3) << 1)) << 4);
    }
    if (ROW == 32) {
        const int line = r >> 2;
        return line * 128 + ((((r & 3) << 1 | c) ^ ((line & 1) << 1)) << 4);
    }
    if (ROW == 64) {
        const int line = r >> 1;
        return line * 128 + ((((r & 1) << 2 | c) ^ ((line & 1) << 1 ^ (line & 2) << 1)) << 4);
    }
    return r * ROW + ((c ^ ((r & 3) << 1) ^ ((r >> 2 & 1) * 5)) << 4);
}

// 8 elements of q from element i on, as they stand: one 16-byte word of a 16-bit type, two of fp32 (W)
template <int W>
__device__ __forceinline__ void load_q8(const AttnArg &a, int64_t token, int head, int i, uint4 *v) {
    if (W == 2 && a.q_dtype == WICI_F32) {
        const float *p = a.q.row<float>(token, head) + i;
        if (a.q_wide) {
            v[0] = ((const uint4 *)p)[0];
            v[W - 1] = ((const uint4 *)p)[1];
        } else {
            v[0] = make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
            v[W - 1] = make_uint4(__float_as_uint(p[4]), __float_as_uint(p[5]), __float_as_uint(p[6]), __float_as_uint(p[7]));
        }
        return;
    }
    const uint16_t *p = a.q.row<uint16_t>(token, head) + i;
    if (a.q_wide) {
        v[0] = *(const uint4 *)p;
    } else {
        v[0] = make_uint4(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16, p[4] | (uint32_t)p[5] << 16,
                          p[6] | (uint32_t)p[7] << 16);
    }
}
// those as fp32
template <int W>
__device__ __forceinline__ void unpack_q8(int dtype, const uint4 *v, float *x) {
    if (W == 2 && dtype == WICI_F32) {
        const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[W - 1].x, v[W - 1].y, v[W - 1].z, v[W - 1].w};
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
        return;
    }
    const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (dtype == WICI_BF16) {
            x[2 * j] = bf16lo(w[j]);
            x[2 * j + 1] = bf16hi(w[j]);
        } else {
            const float2 f = __half22float2(*(const __half2 *)&w[j]);
            x[2 * j] = f.x;
            x[2 * j + 1] = f.y;
        }
    }
}
// 4 elements of the result, element by element: heads that are not 16-byte aligned
static __device__ __noinline__ void store_out4_narrow(const HeadsArg &out, int dtype, int64_t token, int head, int i, float4 v) {
    const float f[4] = {v.x, v.y, v.z, v.w};
    for (int j = 0; j < 4; ++j) {
        if (dtype == WICI_F32) out.row<float>(token, head)[i + j] = f[j];
        else if (dtype == WICI_F16) out.row<__half>(token, head)[i + j] = __float2half_rn(f[j]);
        else out.row<__nv_bfloat16>(token, head)[i + j] = __float2bfloat16_rn(f[j]);
    }
}
__device__ __forceinline__ void store_out4(const AttnArg &a, int64_t token, int head, int i, const float *v) {
    if (!a.out_wide) {
        store_out4_narrow(a.out, a.out_dtype, token, head, i, make_float4(v[0], v[1], v[2], v[3]));
    } else if (a.out_dtype == WICI_F32) {
        *(float4 *)(a.out.row<float>(token, head) + i) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        uint2 w;
        if (a.out_dtype == WICI_F16) {
            const __half2 lo = __floats2half2_rn(v[0], v[1]), hi = __floats2half2_rn(v[2], v[3]);
            w = make_uint2(*(const uint32_t *)&lo, *(const uint32_t *)&hi);
        } else {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
            w = make_uint2(*(const uint32_t *)&lo, *(const uint32_t *)&hi);
        }
        *(uint2 *)(a.out.row<uint16_t>(token, head) + i) = w;
    }
}

// the keys of a sequence: [lo, n), none where the length is bad or not positive
struct Keys {
    int lo, n;
};
__device__ __forceinline__ Keys keys_of(int length, int window) {
    return Keys{window && length > window ? length - window : 0, length};
}

template <int FMT, int D, bool STACK, bool EXACT>
__global__ void __launch_bounds__(kAttnThreads, AttnShape<FMT, D, STACK>::kBlocks) paged_attention_kernel(const __grid_constant__ AttnArg a) {
    using S = AttnShape<FMT, D, STACK>;
    constexpr bool BF16 = FMT == WICI_KV_BF16;
    constexpr bool E2M1 = FMT == WICI_KV_E2M1;
    constexpr int ROW = kv_row_bytes(FMT, D);             // bytes of a key row
    constexpr int CHUNKS = ROW / 16;
    constexpr int TAIL = (S::kBlock - kKvPage * ROW) / 16;   // 16-byte words of a block behind its rows: scales
    constexpr int P = S::kPages, UNIT = P * kKvPage;      // keys of a unit
    constexpr int HT = S::kRows;
    constexpr int R = STACK ? 1 : 2;                      // queries whose rows a lane holds
    constexpr int TQ = !EXACT ? 1 : BF16 ? 3 : 2;
    constexpr int TP = BF16 && EXACT ? 3 : 2;
    constexpr int QPASS = STACK ? (TQ + 1) / 2 : TQ, PPASS = STACK ? (TP + 1) / 2 : TP;
    constexpr int STEPS = D / 16, NT = D / 8;
    constexpr int SETS = P == 1 ? 2 : 1;                  // accumulators of a score: four chains of products at least
    constexpr int KS = S::kKSlots, VS = S::kVSlots;
    constexpr int PER = BF16 || D == 64 ? 8 : 16;         // adjacent elements of O that a lane holds per column
    // The reference of a row's exponents moves when a score passes it by more than kLag (base 2): moving it
    // rescales all of O, which a new maximum would ask for in about 24 of a run's first 60 units (random scores, 16
    // rows of which any may rise), one that far above the last hardly ever.
    constexpr float kLag = 6.f;
    // 8-bit: a row's weights are multiplied by a power of two that takes the largest so far to at most 2^8 when it is
    // chosen, and is chosen again when one passes 2^15: fp16 holds 2^16, and 2^-25 as the second term's last half bit.
    constexpr float kPRoom = 256.f, kPMost = 0x1p15f;

    extern __shared__ __align__(128) uint8_t smem[];
    struct Rec {                          // a segment
        uint32_t start, end;              // units
        int b, head;                      // head: of HH
    };
    struct Shared {
        Rec leaving[kAttnWarps];          // the segment that goes on past a warp's run (end = 0: none)
        Rec side[2];                      // the one that enters the block's run, the one that begins in it and leaves it
        int first[2], last[2];            // blocks that share it
        int note[kAttnWarps];
    };
    static_assert(sizeof(Shared) <= 128, "counted in kSmem");
    uint8_t *parts = smem + kAttnWarps * S::kRing;                    // of warps 1.. : the part that ends in its run
    Shared &sh = *(Shared *)(parts + (kAttnWarps - 1) * S::kPart);
    int *prefix = (int *)((uint8_t *)&sh + 128);                      // [batch + 1]: units of a head before a sequence
    int *weight = prefix + S::kMaxBatch + 1;                         // [batch + 1]: the same with their segments' weights
    int *length = weight + S::kMaxBatch + 1;                         // [batch]

    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * S::kRing;
    griddep_launch_dependents();
    griddep_wait();

    // ---- units of every sequence, and their sums ----
    {
        const int per = (a.batch + kAttnThreads - 1) / kAttnThreads;
        const int b0 = min(a.batch, (int)threadIdx.x * per), b1 = min(a.batch, b0 + per);
        int sum = 0, segments = 0;
        for (int b = b0; b < b1; ++b) {
            int n = a.lengths[b];
            if (n > a.max_pages * (int64_t)kKvPage) n = -1;
            else if (n < 0) n = 0;
            length[b] = n;                               // -1: too long for its row of pages
            const Keys k = keys_of(n, a.window);
            const int units = k.n > 0 ? ((k.n + kKvPage - 1) / kKvPage - k.lo / kKvPage + P - 1) / P : 0;
            prefix[b] = units;
            sum += units;
            segments += units > 0;
        }
        int incl = sum, incl_s = segments;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o), v_s = __shfl_up_sync(0xffffffffu, incl_s, o);
            if (lane >= o) incl += v, incl_s += v_s;
        }
        if (lane == 31) sh.note[warp] = incl;
        int *count_s = (int *)sh.leaving;                // free until the runs are known
        if (lane == 31) count_s[warp] = incl_s;
        __syncthreads();
        int at = incl - sum, at_s = incl_s - segments;
        for (int w = 0; w < warp; ++w) at += sh.note[w], at_s += count_s[w];
        for (int b = b0; b < b1; ++b) {
            const int units = prefix[b];
            prefix[b] = at;
            weight[b] = at + kAttnSegment * at_s;
            at += units;
            at_s += units > 0;
        }
        if (b1 == a.batch) {
            prefix[a.batch] = at;
            weight[a.batch] = at + kAttnSegment * at_s;
        }
        __syncthreads();
    }
    const uint32_t HH = a.cache.kv_heads * a.tiles;
    const uint32_t V = weight[a.batch] * HH;             // weight of all segments: below 2^31

    // ---- this block's run of units, and this warp's ----
    // (a whole number of blocks for each head where there are more: equally long segments then share no block)
    // (e2m1: a unit's work is worth a part of its own: 8 sequences of 1000 tokens, 5 queries a KV head 13.8 us, 15.2 with 2)
    constexpr uint32_t MIN = E2M1 ? 1 : kAttnMinUnits;
    uint32_t blocks = min(gridDim.x, (V + kAttnWarps * MIN - 1) / (kAttnWarps * MIN));
    if (blocks > HH) blocks -= blocks % HH;
    // sequences without keys: zeros, or NaN where the length is bad.  The last blocks begin: with few units they have none.
    for (int b = gridDim.x - 1 - blockIdx.x; b < a.batch; b += gridDim.x) {
        if (prefix[b + 1] != prefix[b]) continue;
        const bool bad = length[b] < 0;
        const float fill = bad ? __uint_as_float(0x7FC00000u) : 0.f, f4[4] = {fill, fill, fill, fill};
        for (int i = threadIdx.x; i < a.q_heads * (D / 4); i += kAttnThreads)
            store_out4(a, b, i / (D / 4), i % (D / 4) * 4, f4);
        if (a.lse)
            for (int h = threadIdx.x; h < a.q_heads; h += kAttnThreads)
                a.lse[(int64_t)b * a.q_heads + h] = bad ? fill : -INFINITY;
        if (bad && threadIdx.x == 0 && a.status) atomicOr(a.status, WICI_BAD_LENGTH);
    }
    if (blockIdx.x >= blocks) return;

    // the last b with sums[b] <= q: it has units (sums[lo] <= q < sums[hi])
    auto last_at = [&](const int *sums, int q, int lo, int hi) {
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (sums[mid] <= q) lo = mid; else hi = mid;
        }
        return lo;
    };
    auto segment_at = [&](uint32_t u) {            // the one that unit u is of
        Rec s;
        s.b = last_at(prefix, u / HH, 0, a.batch);
        const uint32_t n_b = prefix[s.b + 1] - prefix[s.b], r = u - prefix[s.b] * HH;
        s.head = r / n_b;
        s.start = u - (r - s.head * n_b);
        s.end = s.start + n_b;
        return s;
    };
    // Blocks' runs are cut where the weight is: block j of n begins at weight floor(j V / n), or, in a segment of
    // little weight, at the nearer end of it: such a segment then needs no other block's piece.
    const uint32_t runs = kAttnWarps * blocks, whole_w = V / runs, rest_w = V - whole_w * runs;
    int edge_b = a.batch;                          // the sequence that it lies in
    uint32_t edge = V;
    {
        const uint32_t j = kAttnWarps * (blockIdx.x + (lane >= kAttnWarps));
        const uint32_t x = j * whole_w + j * rest_w / runs;         // j, rest_w < 2^14
        if (x < V) {
            edge = x;
            edge_b = last_at(weight, x / HH, 0, a.batch);
            const uint32_t n = prefix[edge_b + 1] - prefix[edge_b] + kAttnSegment, y = (x - weight[edge_b] * HH) % n;
            if (n <= kAttnWhole) edge += 2 * y < n ? -y : n - y;
        }
    }
    // a warp's run is a quarter of its block's, in weight
    auto unit_at = [&](uint32_t x, int lo, int hi) {
        if (x >= V) return prefix[a.batch] * HH;
        const int b = last_at(weight, x / HH, lo, hi);
        const uint32_t r = x - weight[b] * HH, n_b = prefix[b + 1] - prefix[b];
        const uint32_t head = r / (n_b + kAttnSegment), y = r - head * (n_b + kAttnSegment);
        return prefix[b] * HH + head * n_b + (y > kAttnSegment ? y - kAttnSegment : 0u);
    };
    // the block whose run holds unit s.start + z of a segment that several share: of the last run that starts at its
    // weight or before (edges that were moved stay on their side of it)
    auto block_of = [&](const Rec &s, uint32_t z) {
        const uint64_t w = weight[s.b] * HH + s.head * (s.end - s.start + kAttnSegment) + kAttnSegment + z;
        return (int)(((w + 1) * runs - 1) / V / kAttnWarps);
    };
    const uint32_t w0 = __shfl_sync(0xffffffffu, edge, 0), w_run = __shfl_sync(0xffffffffu, edge, kAttnWarps) - w0;
    const int b_first = __shfl_sync(0xffffffffu, edge_b, 0), b_last = __shfl_sync(0xffffffffu, edge_b, kAttnWarps);
    const int part = min(lane, kAttnWarps);
    const uint32_t bound = unit_at(w0 + w_run / kAttnWarps * part + w_run % kAttnWarps * part / kAttnWarps, b_first,
                                   min(a.batch, b_last + 2));
    auto run_at = [&](int w) { return __shfl_sync(0xffffffffu, bound, w); };   // by whole warps
    const uint32_t u0 = run_at(0), u1 = run_at(kAttnWarps), r0 = run_at(warp), r1 = run_at(warp + 1);
    const int mine = (int)(r1 - r0);

    // ---- issue side: lane l knows unit 32 k + l of this warp's ----
    struct Desc {
        int page[P];   // as the table has it; -1 past the sequence's end
        int info;      // kv head | first valid row << 16 | rows end << 24
    };
    auto describe = [&](int i) {
        Desc d;
#pragma unroll
        for (int p = 0; p < P; ++p) d.page[p] = -1;
        d.info = 0;
        if (i >= mine) return d;
        const Rec s = segment_at(r0 + i);
        const int b = s.b, head = s.head, at = (int)(r0 + i - s.start) * P;
        const Keys k = keys_of(length[b], a.window);
        const int first_page = k.lo / kKvPage + at;
        const int32_t *row = a.pages + b * a.table_stride + (int64_t)(head / a.tiles) * a.head_stride;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if ((first_page + p) * (int64_t)kKvPage < k.n) d.page[p] = row[first_page + p];
        }
        const int first = max(0, k.lo - first_page * kKvPage), end = min(UNIT, k.n - first_page * kKvPage);
        d.info = head / a.tiles | first << 16 | end << 24;
        return d;
    };
    Desc cur = describe(lane), next = describe(32 + lane);
    int issued = 0;                       // K's of units issued; V's follow one behind
    uint32_t k_to = ring, v_to = ring + KS * S::kSlot;   // their slots
    uint32_t bad_units = 0;               // bit i % 32: unit i has a bad page
    const uint8_t *last_src[P] = {};      // of the unit before: K of its head in each page (null: no page), its rows
    int last_first = 0, last_end = 0;     // (end 0: no unit)

    const uint64_t policy = l2_evict_first();   // read once: code, queries and parts stay in L2 instead
    const uint32_t lane_dst = chunk_at<ROW, E2M1>(lane / CHUNKS, lane % CHUNKS);
    const int64_t lane_v = (int64_t)a.cache.kv_heads * S::kBlock;   // from K to V of a head in a page
    constexpr int N = kKvPage * CHUNKS / 32, ROWS = 32 / CHUNKS;    // a page's block in N rounds of the warp, rows of a round
    // a unit's K or V: rows without a key of the sequence are zeroed, what the cache holds there is anything
    auto copy_unit = [&](uint32_t dst, const uint8_t *const *src, int64_t off, int first, int end) {
        if (first == 0 && end == UNIT) {                     // every page is there
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const uint8_t *from = src[p] + off + lane * 16;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    cp_async16(dst + p * S::kBlock + (chunk_at<ROW, E2M1>(i * ROWS, 0) ^ lane_dst), from + i * 512, 16, policy);
                if (lane < TAIL) cp_async16(dst + p * S::kBlock + kKvPage * ROW + lane * 16, from + kKvPage * ROW, 16, policy);
            }
        } else {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const uint8_t *from = src[p] ? src[p] + off + lane * 16 : a.cache.data;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int r = p * kKvPage + i * ROWS + lane / CHUNKS;
                    cp_async16(dst + p * S::kBlock + (chunk_at<ROW, E2M1>(i * ROWS, 0) ^ lane_dst), src[p] ? from + i * 512 : from,
                               src[p] && r >= first && r < end ? 16 : 0, policy);
                }
                if (lane < TAIL)
                    cp_async16(dst + p * S::kBlock + kKvPage * ROW + lane * 16, src[p] ? from + kKvPage * ROW : from,
                               src[p] ? 16 : 0, policy);
            }
        }
    };
    // e2m1: a unit's K or V as it is; of rows without a key nothing is used (their codes are finite numbers whatever they are,
    // their scales are left out).  A page that is not there gives zeros.
    const uint32_t tail_dst = kKvPage * ROW + lane * 16;
    auto copy_whole = [&](uint32_t dst, const uint8_t *const *src, int64_t off) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const uint8_t *from = (src[p] ? src[p] + off : a.cache.data) + lane * 16;
            const int bytes = src[p] ? 16 : 0;
#pragma unroll
            for (int i = 0; i < N; ++i) cp_async16(dst + lane_dst + (p * S::kBlock + i * 512), from + i * 512, bytes, policy);
            cp_async16_if(lane < TAIL, dst + tail_dst + p * S::kBlock, from + kKvPage * ROW, bytes, policy);
        }
    };
    // group j: K of unit j and V of the one before it (none past the last unit: the groups still count)
    auto issue = [&]() {
        if (issued && (issued & 31) == 0) {
            cur = next;
            next = describe(issued + 32 + lane);
        }
        // (e2m1: a unit past the last one has no pages; its zeros go where nothing is read)
        if constexpr (E2M1) {
            if (issued) copy_whole(v_to, last_src, lane_v);
        } else if (last_end) copy_unit(v_to, last_src, lane_v, last_first, last_end);
        if (issued) v_to = v_to == ring + (KS + VS - 1) * S::kSlot ? ring + KS * S::kSlot : v_to + S::kSlot;
        last_end = 0;
        if (E2M1 || issued < mine) {
            const int info = __shfl_sync(0xffffffffu, cur.info, issued & 31);
            int first = info >> 16 & 255, end = info >> 24;
            const uint8_t *head = a.cache.data + (int64_t)((info & 0xFFFF) * S::kBlock);
            bool bad = false;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int page = __shfl_sync(0xffffffffu, cur.page[p], issued & 31);
                const bool there = (uint32_t)page < (uint32_t)a.cache.n_pages;
                bad |= !there && end > p * kKvPage;          // one that the sequence needs
                last_src[p] = there ? head + page * a.cache.page_stride : nullptr;
            }
            if (bad) {
                bad_units |= 1u << (issued & 31);
                if (lane == 0 && a.status) atomicOr(a.status, WICI_BAD_PAGE);
                first = -1;                                  // not the way of whole units
            }
            if constexpr (E2M1) copy_whole(k_to, last_src, 0);
            else copy_unit(k_to, last_src, 0, first, end);
            last_first = first;
            last_end = end;
        }
        k_to = k_to == ring + (KS - 1) * S::kSlot ? ring : k_to + S::kSlot;
        ++issued;
        cp_commit();
    };

    // ---- segments of this warp's run ----
    Rec seg = {r0, r0, 0, 0};
    if (mine > 0) seg = segment_at(r0);
    constexpr int QW = EXACT ? 2 : 1;     // 16-byte words of 8 elements of q: fp32 comes with EXACT alone
    uint4 qx[R][STEPS / 2][QW];           // the segment's queries
    auto load_queries = [&]() {
        const int row0 = seg.head % a.tiles * HT, head0 = seg.head / a.tiles * a.group + row0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < STEPS / 2; ++i) {
                // a step takes 4 adjacent elements of a lane's chunk: bf16 of chunk 4 i + t, 8-bit of half i % 2 of 4 (i / 2) + t
                const int e0 = BF16 ? 8 * (4 * i + t) : 16 * (4 * (i / 2) + t) + 8 * (i % 2);
#pragma unroll
                for (int w = 0; w < QW; ++w) qx[r][i][w] = make_uint4(0, 0, 0, 0);
                if (g + 8 * r < a.group - row0) load_q8<QW>(a, seg.b, head0 + g + 8 * r, e0, qx[r][i]);
            }
    };
    if (mine > 0) load_queries();         // before the ring's copies, which queue up in front of what comes after
#pragma unroll 1
    for (int i = 0; i < KS; ++i) issue();
    // while they are on their way: who shares the segments at the block's ends
    if (lane == 0) sh.leaving[warp].end = 0;
    if (warp < 2) {
        Rec s = {0, 0, 0, 0};
        if (u0 < u1) s = segment_at(warp ? u1 - 1 : u0);   // a block may have got the weight of a segment and none of its units
        if (warp ? s.end <= u1 || s.start < u0 : s.start >= u0) s.end = 0;
        else if (lane == 0) sh.first[warp] = block_of(s, 0), sh.last[warp] = block_of(s, s.end - s.start - 1);
        if (lane == 0) sh.side[warp] = s;
    }

    // a part of a segment: rows of O (kPartRow floats each), then m and l of each row
    auto part_of = [&](int w, bool last_of_run) {
        return (float *)(last_of_run ? smem + w * S::kRing : parts + (w - 1) * S::kPart);
    };
    int done = 0;                         // units of this warp computed
    uint32_t ks = ring, vs = ring + KS * S::kSlot;       // slots of the next one to compute
    while (done < mine) {
        const int stop = (int)(min(seg.end, r1) - r0);
        const Keys keys = keys_of(length[seg.b], a.window);
        const int row0 = seg.head % a.tiles * HT, rows = min(HT, a.group - row0);   // first query of the tile in the group
        const int head0 = seg.head / a.tiles * a.group + row0, seg_b = seg.b;

        // where the part of a segment that this run shares goes, and its rows' m and l
        struct Part {
            float *at;
            int row;
            float2 *ml;
        };
        auto leave = [&](bool left) {
            if (left) {
                cp_wait<0>();                               // the ring is free: no unit follows
                if (lane == 0) sh.leaving[warp] = seg;
            }
            __syncwarp();
            // what ends in the block's first run is the block's whole part of its segment
            const bool to_piece = !left && r0 == u0;
            Part p;
            p.at = to_piece ? a.pieces + (int64_t)blockIdx.x * 2 * attn_piece_floats(D) : part_of(warp, left);
            p.row = to_piece ? D : S::kPartRow;
            p.ml = (float2 *)(p.at + (to_piece ? kAttnPieceRows * D : HT * S::kPartRow));
            return p;
        };

        if constexpr (E2M1) {
            // ==== keys are the rows of S^T = K Q^T, elements of the head those of O^T = V^T P^T, queries the columns of
            // both: a lane has keys g and g + 8 of a page for queries 2 t and 2 t + 1 of each tile of 8 (N8 of them).  Two
            // terms of q or p are two products into the same sums, so O takes half of the registers that rows for each term
            // would, and the codes, whose conversion costs most here, are converted once for both ====
            constexpr int N8 = R, C = 2 * N8, TILES = D / 16;
            constexpr int J = 2 * P;                          // keys of a query that a lane has
            constexpr int EACH_AT = kKvPage * ROW, SCALES_AT = kv_scales_at(FMT, D);

            // ---- Q fragments: query g of a tile, 4 elements a step ----
            uint32_t qf[N8][TQ][STEPS][2];
            float cq[C];                                      // products to base-2 logits, of queries 2 t, 2 t + 1
            const float log2_scale = a.scale * 1.44269504088896340736f;
            // the smallest power of two that takes the scale to no less than 2^-126, where it has its 24 bits (what smaller
            // queries lose by it is below head_dim 2^-25 2^-126 max|k| < 2^-16 of a logit)
            const int least = 1 - min((int)(__float_as_uint(log2_scale) >> 23 & 0xFF), 127);
#pragma unroll
            for (int n = 0; n < N8; ++n) {
                float x[STEPS][4];
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < STEPS / 2; ++i) unpack_q8<QW>(a.q_dtype, qx[n][i], x[2 * i]);
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(x[s][j]) & 0x7FFFFFFFu);
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // 2^(13 - exponent): the largest magnitude to [2^13, 2^14), a smaller one where q and the scale are very small
                int e = (int)(top >> 23) - 127 - 13;
                e = top >= kInfBits ? 0 : max(least, e);
                const float down = __int_as_float((127 - e) << 23), of_g = log2_scale * __int_as_float((127 + e) << 23);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    uint32_t w[2][TQ];
                    split<false, false, false, TQ>(x[s][0] * down, x[s][1] * down, w[0], 1.f);
                    split<false, false, false, TQ>(x[s][2] * down, x[s][3] * down, w[1], 1.f);
#pragma unroll
                    for (int k = 0; k < TQ; ++k) qf[n][k][s][0] = w[0][k], qf[n][k][s][1] = w[1][k];
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) cq[2 * n + j] = __shfl_sync(0xffffffffu, of_g, 4 * (2 * t + j));
            }

            float m[C], l[C], o[TILES][N8][4], heaviest[C], per[C];   // the largest weight so far, what weights are multiplied by
#pragma unroll
            for (int r = 0; r < C; ++r) m[r] = -INFINITY, l[r] = 0.f, heaviest[r] = 0.f, per[r] = kPRoom * 0x1p118f;
#pragma unroll
            for (int x = 0; x < TILES; ++x)
#pragma unroll
                for (int n = 0; n < N8; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[x][n][j] = 0.f;
            // O so far is multiplied by f for `per` to follow `heaviest`
            auto follow = [&](int r, float f) {
                const float was = __uint_as_float(0x7F000000u - __float_as_uint(per[r])) * f;      // f / per
                const uint32_t e = min(max((__float_as_uint(heaviest[r]) + 0x7FFFFFu) & 0x7F800000u, 0x04800000u), 0x7E800000u);
                per[r] = kPRoom * __uint_as_float(0x7F000000u - e);      // heaviest to its power of two, in [2^-118, 2^126]
                return was * per[r];
            };
            auto rescale = [&](const float *f) {
#pragma unroll
                for (int x = 0; x < TILES; ++x)
#pragma unroll
                    for (int n = 0; n < N8; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[x][n][j] *= f[2 * n + (j & 1)];
            };
            auto largest = [&](float v) {                     // of the 8 lanes that share queries
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
                return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
            };
            auto key_at = [&](int j) { return (j >> 1) * kKvPage + (j & 1) * 8 + g; };

            // where a lane's parts of a block are: of K the chunk t of key g (chunk 4 + t is 32 bytes across, key g + 8 as far
            // on as rows are), of V the chunk g of key 2 t (key 2 t + 1 is ODD bytes across), and their block scales
            constexpr uint32_t ODD = D == 128 ? 64 : 32, EIGHT = 8 * ROW;
            const uint32_t k_lane = chunk_at<ROW, E2M1>(g, t >> 1) + (t & 1) * 8, each_k = EACH_AT + g * (D / 16) + t;
            const uint32_t v_lane = D == 128 ? chunk_at<ROW, E2M1>(2 * t, g >> 1) + (g & 1) * 8 : chunk_at<ROW, E2M1>(2 * t, g >> 2) + (g & 3) * 4;
            const uint32_t each_v = EACH_AT + 2 * t * (D / 16) + (D == 128 ? g : g >> 1);

            // ---- scores of one unit (unscaled) ----
            float c[P][N8][4];
            auto scores = [&](uint32_t slot) {
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
#pragma unroll
                    for (int pg = 0; pg < P; ++pg) {
                        uint32_t h[2][8], b[2];               // 16 elements of keys g, g + 8: 8 bytes and a scale
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint2 w = lds64(slot + (i ? k_lane ^ 32 : k_lane) + pg * S::kBlock + k * EIGHT);
                            b[k] = e4m3_half(lds8(slot + each_k + pg * S::kBlock + k * (D / 2) + 4 * i));
                            decode_e2m1(w.x, h[k]);
                            decode_e2m1(w.y, h[k] + 4);
                        }
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            const uint32_t f[4] = {times_low(h[0][2 * s], b[0]), times_low(h[1][2 * s], b[1]),
                                                   times_low(h[0][2 * s + 1], b[0]), times_low(h[1][2 * s + 1], b[1])};
#pragma unroll
                            for (int n = 0; n < N8; ++n)
#pragma unroll
                                for (int k = 0; k < TQ; ++k) mma_f16(c[pg][n], i == 0 && s == 0 && k == 0, f, qf[n][k][4 * i + s]);
                        }
                    }
                }
            };

            // ---- units of this segment: the scores of the next one run beside the softmax of this one (past the last
            // one they are not used, whatever the slot holds) ----
            int key0 = (keys.lo / kKvPage + (int)(r0 + done - seg.start) * P) * kKvPage;   // first key of the unit
            cp_wait<KS - 1>();                                // group `done` brings its K
            __syncwarp();
            scores(ks);
            for (; done < stop; ++done, key0 += UNIT) {
                // group done + 1: K of the next unit and V of this one
                cp_wait<KS - 2>();
                __syncwarp();
                const uint32_t ks_next = ks == ring + (KS - 1) * S::kSlot ? ring : ks + S::kSlot;
                float x[C][J];                                // queries 2 t + r % 2 of tile r / 2, keys key_at(j)
                const bool part = key0 < keys.lo || key0 > keys.n - UNIT;   // not every key of the unit is the sequence's
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const float ksc = lds32(ks + (j >> 1) * S::kBlock + SCALES_AT + (j & 1) * 32 + 4 * g);
                    // Rounded here, once for the reference and for the exponent, which is 0 then for the largest logit: a product
                    // taken into the exponent's own rounding is off from the reference by up to 2^-25 of a logit of any size.
                    // (c is up to 2^32, of a query scaled to 2^13: cq's power of two goes to the key's scale, which may be 2^116, first.)
#pragma unroll
                    for (int r = 0; r < C; ++r) x[r][j] = __fmul_rn(c[j >> 1][r >> 1][2 * (j & 1) + (r & 1)], ksc * cq[r]);
                }
                if (part) {
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const int key = key0 + key_at(j);
#pragma unroll
                        for (int r = 0; r < C; ++r) x[r][j] = key >= keys.lo && key < keys.n ? x[r][j] : -INFINITY;
                    }
                }
                float up[C];
                bool grew = false;
#pragma unroll
                for (int r = 0; r < C; ++r) {
                    float top = x[r][0];
#pragma unroll
                    for (int j = 1; j < J; ++j) top = fmaxf(top, x[r][j]);
                    up[r] = fmaxf(m[r], largest(top));
                    grew |= up[r] > m[r] + kLag;
                }
                if (__any_sync(0xffffffffu, grew)) {
                    float f[C];
#pragma unroll
                    for (int r = 0; r < C; ++r) {
                        f[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - up[r]);   // nothing yet: zeros
                        l[r] *= f[r];
                        m[r] = up[r];
                        heaviest[r] *= f[r];
                        f[r] = follow(r, f[r]);
                    }
                    rescale(f);
                }
                scores(ks_next);                              // c has been read
                // the weights in the place of the scores
                bool heavy = false;
                float ref[C], top[C];
#pragma unroll
                for (int r = 0; r < C; ++r) ref[r] = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const float vscale = lds32(vs + (j >> 1) * S::kBlock + SCALES_AT + (j & 1) * 32 + 4 * g);
#pragma unroll
                    for (int r = 0; r < C; ++r) {
                        const float p = ex2(x[r][j] - ref[r]);
                        l[r] += p;
                        x[r][j] = p * vscale;
                    }
                }
                if (part) {                                   // scales of other keys may be anything
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const int key = key0 + key_at(j);
#pragma unroll
                        for (int r = 0; r < C; ++r) x[r][j] = key >= keys.lo && key < keys.n ? x[r][j] : 0.f;
                    }
                }
#pragma unroll
                for (int r = 0; r < C; ++r) {
                    top[r] = x[r][0];
#pragma unroll
                    for (int j = 1; j < J; ++j) top[r] = fmaxf(top[r], x[r][j]);
                    heavy |= top[r] * per[r] > kPMost;
                }
                if (__any_sync(0xffffffffu, heavy)) {
                    float f[C];
#pragma unroll
                    for (int r = 0; r < C; ++r) {
                        heaviest[r] = largest(fmaxf(heaviest[r], top[r]));
                        f[r] = follow(r, 1.f);
                    }
                    rescale(f);
                }
                // EXACT (fp32): a unit's sums apart, added to O in fp32: in one sum the tensor cores' cut additions make 4096 keys
                // 2.1e-6 too small (7e-7 off this way; head_dim 64 42.2 and 42.7 us, 128 61.7 and 65.7)
                float sum[TILES][N8][4];
#pragma unroll
                for (int pg = 0; pg < P; ++pg) {
                    uint32_t pf[N8][2][2];                    // [tile][term][keys 0..7, 8..15]
#pragma unroll
                    for (int n = 0; n < N8; ++n)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            uint32_t w[2];
                            split<false, false, true, 2>(x[2 * n][2 * pg + k] * per[2 * n], x[2 * n + 1][2 * pg + k] * per[2 * n + 1], w, 1.f);
                            pf[n][0][k] = transposed(w[0]);
                            pf[n][1][k] = transposed(w[1]);
                        }
                    // V: keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9; element 2 x of the lane's PER is row g of tile x, the next row g + 8
                    constexpr int WORDS = D / 64;             // 4-byte words of a row that a lane takes
                    const uint32_t vp = vs + pg * S::kBlock;
                    uint32_t w[4][WORDS], b[4], b2[2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t at = vp + (i & 1 ? v_lane ^ ODD : v_lane) + (i >> 1) * EIGHT;
                        if (D == 128) {
                            const uint2 q = lds64(at);
                            w[i][0] = q.x, w[i][WORDS - 1] = q.y;
                        } else {
                            w[i][0] = __float_as_uint(lds32(at));
                        }
                        b[i] = lds8(vp + each_v + ((i & 1) + (i >> 1) * 8) * (D / 16));
                    }
                    if (part) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {         // of another key: may be NaN
                            const int key = key0 + pg * kKvPage + 2 * t + (i & 1) + (i >> 1) * 8;
                            b[i] = key >= keys.lo && key < keys.n ? b[i] : 0u;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const __half2 v = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(b[2 * i] | b[2 * i + 1] << 8), __NV_E4M3));
                        b2[i] = *(const uint32_t *)&v;
                    }
#pragma unroll
                    for (int x8 = 0; x8 < WORDS; ++x8) {
                        // halves of bytes of two rows interleaved first: elements 2 e in even[..][e], 2 e + 1 in odd[..][e]
                        uint32_t even[2][4], odd[2][4];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t u = w[2 * i][x8], v = w[2 * i + 1][x8];
                            decode_e2m1((u & 0x0F0F0F0Fu) | (v << 4 & 0xF0F0F0F0u), even[i]);
                            decode_e2m1((u >> 4 & 0x0F0F0F0Fu) | (v & 0xF0F0F0F0u), odd[i]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t f[4] = {times(even[0][e], b2[0]), times(odd[0][e], b2[0]), times(even[1][e], b2[1]),
                                                   times(odd[1][e], b2[1])};
#pragma unroll
                            for (int n = 0; n < N8; ++n) {
                                float *to = EXACT ? sum[4 * x8 + e][n] : o[4 * x8 + e][n];
#pragma unroll
                                for (int k = 0; k < 2; ++k) mma_f16(to, EXACT && pg == 0 && k == 0, f, pf[n][k]);
                            }
                        }
                    }
                }
                if (EXACT) {
#pragma unroll
                    for (int i = 0; i < TILES; ++i)
#pragma unroll
                        for (int n = 0; n < N8; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[i][n][j] += sum[i][n][j];
                }
                if (bad_units >> (done & 31) & 1) {
                    bad_units &= ~(1u << (done & 31));
#pragma unroll
                    for (int r = 0; r < C; ++r) l[r] = __uint_as_float(0x7FC00000u);
                }
                __syncwarp();                                 // every lane has read the slots
                issue();
                ks = ks_next;
                vs = vs == ring + (KS + VS - 1) * S::kSlot ? ring + KS * S::kSlot : vs + S::kSlot;
            }

            // ---- the segment's state, or this run's part of it: of queries 2 t, 2 t + 1 elements PER g .. PER g + PER - 1 ----
            const bool entered = seg.start < r0, left = seg.end > r1;
            const Part to = leave(left);
#pragma unroll
            for (int r = 0; r < C; ++r) {
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], s);
                const int row = 8 * (r >> 1) + 2 * t + (r & 1);
                const bool alone = !entered && !left;
                const float f = alone ? 1.f / per[r] / l[r] : 1.f / per[r];
                if (row >= rows) continue;
#pragma unroll
                for (int i = 0; i < PER; i += 4) {
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = o[(i + j) / 2][r >> 1][2 * (j & 1) + (r & 1)] * f;
                    if (alone) store_out4(a, seg_b, head0 + row, PER * g + i, v);
                    else *(float4 *)(to.at + row * to.row + PER * g + i) = make_float4(v[0], v[1], v[2], v[3]);
                }
                if (g == 0) {
                    if (!alone) to.ml[row] = make_float2(m[r], l[r]);
                    else if (a.lse) a.lse[(int64_t)seg_b * a.q_heads + head0 + row] = (m[r] + log2f(l[r])) * 0.693147180559945309417f;
                }
            }
        } else {
            // ---- Q fragments ----
            uint32_t qf[QPASS][STEPS][4];
            float cq[R];                      // products to base-2 logits
#pragma unroll
            for (int r = 0; r < R; ++r) {
                cq[r] = a.scale * 1.44269504088896340736f;
                float x[STEPS][4];
#pragma unroll
                for (int i = 0; i < STEPS / 2; ++i) unpack_q8<QW>(a.q_dtype, qx[r][i], x[2 * i]);
                if (!BF16) {
                    uint32_t top = 0;
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
#pragma unroll
                        for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(x[s][j]) & 0x7FFFFFFFu);
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    // 2^(13 - exponent): the largest magnitude to [2^13, 2^14)
                    int e = (int)(top >> 23) - 127 - 13;
                    e = top >= kInfBits ? 0 : max(-126, min(126, e));   // (of zeros the smallest: a factor that is finite)
                    const float down = __int_as_float((127 - e) << 23);
                    cq[r] *= __int_as_float((127 + e) << 23);
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[s][j] *= down;
                }
#pragma unroll
                for (int s = 0; s < STEPS; ++s) split_row<BF16, false, STACK, TQ, STEPS>(x[s], r, &qf[0][s]);
            }

            float m[R], l[R], o[NT][4];
#pragma unroll
            for (int r = 0; r < R; ++r) m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][j] = 0.f;
            float heaviest[R], per[R];                    // 8-bit: the largest weight so far, what weights are multiplied by
#pragma unroll
            for (int r = 0; r < R; ++r) heaviest[r] = 0.f, per[r] = kPRoom * 0x1p118f;
            // O so far is multiplied by f for `per` to follow `heaviest`
            auto follow = [&](int r, float f) {
                const float was = __uint_as_float(0x7F000000u - __float_as_uint(per[r])) * f;      // f / per
                const uint32_t e = min(max((__float_as_uint(heaviest[r]) + 0x7FFFFFu) & 0x7F800000u, 0x04800000u), 0x7E800000u);
                per[r] = kPRoom * __uint_as_float(0x7F000000u - e);      // heaviest to its power of two, in [2^-118, 2^126]
                return was * per[r];
            };

            // ---- scores of one unit (unscaled) ----
            float c[2 * P][SETS][4];                             // [8 keys][sets of steps]
            auto scores = [&](uint32_t ks) {
#pragma unroll
                for (int n = 0; n < 2 * P; ++n)
#pragma unroll
                    for (int e = 0; e < SETS; ++e)
#pragma unroll
                        for (int j = 0; j < 4; ++j) c[n][e][j] = 0.f;
#pragma unroll
                for (int i = 0; i < CHUNKS / 4; ++i) {
#pragma unroll
                    for (int n = 0; n < 2 * P; ++n) {
                        const int r = (g >> 1) + (g & 1) * 4 + 8 * (n & 1);   // the key of column g
                        const uint4 w = lds128(ks + n / 2 * S::kBlock + chunk_at<ROW, E2M1>(r, 4 * i + t));
                        if (BF16) {
#pragma unroll
                            for (int k = 0; k < QPASS; ++k) {
                                mma16816<true>(c[n][0], qf[k][2 * i], w.x, w.y);
                                mma16816<true>(c[n][SETS - 1], qf[k][2 * i + 1], w.z, w.w);
                            }
                        } else {
                            const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                            for (int s = 0; s < 4; ++s) {
                                uint32_t b0, b1;
                                decode4<FMT>(word[s], b0, b1);
#pragma unroll
                                for (int k = 0; k < QPASS; ++k) mma16816<false>(c[n][0], qf[k][4 * i + s], b0, b1);
                            }
                        }
                    }
                }
            };

            // ---- units of this segment: the scores of the next one run beside the softmax of this one (past the last
            // one they are not used, whatever the slot holds) ----
            int key0 = (keys.lo / kKvPage + (int)(r0 + done - seg.start) * P) * kKvPage;   // first key of the unit
            cp_wait<KS - 1>();                                   // group `done` brings its K
            __syncwarp();
            scores(ks);
            for (; done < stop; ++done, key0 += UNIT) {
                // group done + 1: K of the next unit and V of this one
                cp_wait<KS - 2>();
                __syncwarp();
                const uint32_t ks_next = ks == ring + (KS - 1) * S::kSlot ? ring : ks + S::kSlot;
                // x[r][j]: query g + 8 r, key t + 4 j of the unit
                constexpr int J = 4 * P;
                float x[R][J];
                const bool part = key0 < keys.lo || key0 > keys.n - UNIT;   // not every key of the unit is the sequence's
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int n = j >> 1, col = j & 1;
                    const float ksc = BF16 ? 1.f : lds32(ks + j / 4 * S::kBlock + kKvPage * D + (t + 4 * (j & 3)) * 4);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        float dot = c[n][0][col + 2 * r];
                        if (SETS == 2) dot += c[n][SETS - 1][col + 2 * r];
                        if (STACK && TQ > 1) {
                            dot += c[n][0][col + 2];
                            if (SETS == 2) dot += c[n][SETS - 1][col + 2];
                        }
                        x[r][j] = dot * (BF16 ? cq[r] : ksc * cq[r]);
                    }
                }
                if (part) {
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const int key = key0 + t + 4 * j;
#pragma unroll
                        for (int r = 0; r < R; ++r) x[r][j] = key >= keys.lo && key < keys.n ? x[r][j] : -INFINITY;
                    }
                }
                float up[R];
                bool grew = false;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float top = x[r][0];
#pragma unroll
                    for (int j = 1; j < J; ++j) top = fmaxf(top, x[r][j]);
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    up[r] = fmaxf(m[r], top);
                    grew |= up[r] > m[r] + kLag;
                }
                if (__any_sync(0xffffffffu, grew)) {
                    float f[R];
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        f[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - up[r]);   // nothing yet: zeros
                        l[r] *= f[r];
                        m[r] = up[r];
                        if (!BF16) {
                            heaviest[r] *= f[r];
                            f[r] = follow(r, f[r]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        o[n][0] *= f[0];
                        o[n][1] *= f[0];
                        o[n][2] *= f[R - 1];
                        o[n][3] *= f[R - 1];
                    }
                }
                scores(ks_next);                                 // c has been read
                float ref[R];
#pragma unroll
                for (int r = 0; r < R; ++r) ref[r] = m[r] == -INFINITY ? 0.f : m[r];
                if (!BF16) {
                    // the weights in the place of the scores
                    float top[R];
                    bool heavy = false;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const float vscale = lds32(vs + j / 4 * S::kBlock + kKvPage * D + (t + 4 * (j & 3)) * 4);
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const float p = ex2(x[r][j] - ref[r]);
                            l[r] += p;
                            x[r][j] = p * vscale;
                        }
                    }
                    if (part) {                                  // scales of other keys may be anything
#pragma unroll
                        for (int j = 0; j < J; ++j) {
                            const int key = key0 + t + 4 * j;
#pragma unroll
                            for (int r = 0; r < R; ++r) x[r][j] = key >= keys.lo && key < keys.n ? x[r][j] : 0.f;
                        }
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        top[r] = x[r][0];
#pragma unroll
                        for (int j = 1; j < J; ++j) top[r] = fmaxf(top[r], x[r][j]);
                        heavy |= top[r] * per[r] > kPMost;
                    }
                    if (__any_sync(0xffffffffu, heavy)) {
                        float f[R];
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            heaviest[r] = fmaxf(heaviest[r], top[r]);
                            heaviest[r] = fmaxf(heaviest[r], __shfl_xor_sync(0xffffffffu, heaviest[r], 1));
                            heaviest[r] = fmaxf(heaviest[r], __shfl_xor_sync(0xffffffffu, heaviest[r], 2));
                            f[r] = follow(r, 1.f);
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            o[n][0] *= f[0];
                            o[n][1] *= f[0];
                            o[n][2] *= f[R - 1];
                            o[n][3] *= f[R - 1];
                        }
                    }
                }
                uint32_t pf[P][PPASS][4];
#pragma unroll
                for (int r = 0; r < R; ++r) {
#pragma unroll
                    for (int pg = 0; pg < P; ++pg) {
                        float p[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (BF16) {
                                p[j] = ex2(x[r][4 * pg + j] - ref[r]);
                                l[r] += p[j];
                            } else {
                                p[j] = x[r][4 * pg + j] * per[r];
                            }
                        }
                        split_row<BF16, true, STACK, TP, 1>(p, r, pf[pg]);
                    }
                }
                // V: rows t + 4 i of a page; column g of tile n is element PER (g + 8 (n / PER)) + n % PER of the head
#pragma unroll
                for (int pg = 0; pg < P; ++pg) {
                    const uint32_t vp = vs + pg * S::kBlock;
                    if (BF16) {
#pragma unroll
                        for (int jj = 0; jj < CHUNKS / 8; ++jj) {
                            uint32_t w[4][4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint4 q = lds128(vp + chunk_at<ROW, E2M1>(t + 4 * i, g + 8 * jj));
                                w[i][0] = q.x, w[i][1] = q.y, w[i][2] = q.z, w[i][3] = q.w;
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const uint32_t sel = e & 1 ? 0x7632 : 0x5410;
                                const uint32_t b0 = __byte_perm(w[0][e / 2], w[1][e / 2], sel);
                                const uint32_t b1 = __byte_perm(w[2][e / 2], w[3][e / 2], sel);
#pragma unroll
                                for (int k = 0; k < PPASS; ++k) mma16816<true>(o[8 * jj + e], pf[pg][k], b0, b1);
                            }
                        }
                    } else {
                        constexpr int WORDS = D / 32;          // 4-byte words of a row that a lane takes
                        uint32_t w[4][WORDS];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (D == 128) {
                                const uint4 q = lds128(vp + chunk_at<ROW, E2M1>(t + 4 * i, g));
                                w[i][0] = q.x, w[i][1] = q.y, w[i][WORDS - 2] = q.z, w[i][WORDS - 1] = q.w;
                            } else {
                                const uint2 q = lds64(vp + chunk_at<ROW, E2M1>(t + 4 * i, g >> 1) + (g & 1) * 8);
                                w[i][0] = q.x, w[i][1] = q.y;
                            }
                        }
#pragma unroll
                        for (int x4 = 0; x4 < WORDS; ++x4) {
                            // the bytes of two rows interleaved first: a pair of them is a fragment's half
                            uint32_t h[2][4];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                decode4<FMT>(__byte_perm(w[2 * i][x4], w[2 * i + 1][x4], 0x5140), h[i][0], h[i][1]);
                                decode4<FMT>(__byte_perm(w[2 * i][x4], w[2 * i + 1][x4], 0x7362), h[i][2], h[i][3]);
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int k = 0; k < PPASS; ++k) mma16816<false>(o[4 * x4 + e], pf[pg][k], h[0][e], h[1][e]);
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
                ks = ks_next;
                vs = vs == ring + (KS + VS - 1) * S::kSlot ? ring + KS * S::kSlot : vs + S::kSlot;
            }

            // ---- the segment's state, or this run's part of it ----
            const bool entered = seg.start < r0, left = seg.end > r1;
            const Part to = leave(left);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
                const int row = g + 8 * r;
                const bool alone = !entered && !left;
                const float unit_of_o = BF16 ? 1.f : 1.f / per[r], f = alone ? unit_of_o / l[r] : unit_of_o;
                if (row >= rows) continue;
#pragma unroll
                for (int n = 0; n < NT; n += 4) {
                    // columns 2 t and 2 t + 1 of tiles n .. n + 3: four adjacent elements each
                    float v[2][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < 2; ++c) v[c][i] = (STACK ? rows_sum(o[n + i][c], o[n + i][c + 2]) : o[n + i][2 * r + c]) * f;
                    const int d0 = PER * (2 * t + 8 * (n / PER)) + n % PER;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (alone) store_out4(a, seg_b, head0 + row, d0 + PER * c, v[c]);
                        else *(float4 *)(to.at + row * to.row + d0 + PER * c) = make_float4(v[c][0], v[c][1], v[c][2], v[c][3]);
                    }
                }
                if (t == 0) {
                    if (!alone) to.ml[row] = make_float2(m[r], l[r]);
                    else if (a.lse) a.lse[(int64_t)seg_b * a.q_heads + head0 + row] = (m[r] + log2f(l[r])) * 0.693147180559945309417f;
                }
            }
        }
        if (seg.end < r1) {
            seg.start = seg.end;
            if (++seg.head == (int)HH) {
                seg.head = 0;
                do ++seg.b; while (prefix[seg.b + 1] == prefix[seg.b]);
            }
            seg.end = seg.start + prefix[seg.b + 1] - prefix[seg.b];
            load_queries();
        }
    }
    cp_wait<0>();
    __syncthreads();

    // ---- segments that several runs share ----
    auto rows_of = [&](const Rec &s) { return min(HT, a.group - s.head % a.tiles * HT); };
    auto finish = [&](const Rec &s, int row, int d0, const float *v, float top, float sum) {
        const int head = s.head / a.tiles * a.group + s.head % a.tiles * HT + row;
        const float inv = 1.f / sum, q[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
        store_out4(a, s.b, head, d0, q);
        if (d0 == 0 && a.lse) a.lse[(int64_t)s.b * a.q_heads + head] = (top + log2f(sum)) * 0.693147180559945309417f;
    };
    uint32_t run[kAttnWarps + 1];
#pragma unroll
    for (int w = 0; w <= kAttnWarps; ++w) run[w] = run_at(w);
    uint32_t joined = ~0u;                // start of the segment joined last
#pragma unroll
    for (int w = 0; w < kAttnWarps; ++w) {
        const Rec s = sh.leaving[w];
        if (s.end == 0 || s.start == joined) continue;
        joined = s.start;
        // its parts: of warp w, then of the runs after it up to the one where it ends
        const bool whole = s.start >= u0 && s.end <= u1;
        float *piece = a.pieces + ((int64_t)blockIdx.x * 2 + (s.start >= u0 ? 1 : 0)) * attn_piece_floats(D);
        for (int i = threadIdx.x; i < rows_of(s) * (D / 4); i += kAttnThreads) {
            const int row = i / (D / 4), d0 = i % (D / 4) * 4;
            float top = -INFINITY, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = w; x < kAttnWarps; ++x)
                if (run[x] < run[x + 1] && run[x] < s.end)
                    top = fmaxf(top, ((const float2 *)(part_of(x, s.end > run[x + 1]) + HT * S::kPartRow))[row].x);
#pragma unroll
            for (int x = w; x < kAttnWarps; ++x) {
                if (run[x] == run[x + 1] || run[x] >= s.end) continue;
                const float *src = part_of(x, s.end > run[x + 1]);
                const float2 ml = ((const float2 *)(src + HT * S::kPartRow))[row];
                const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
                const float4 q = *(const float4 *)(src + row * S::kPartRow + d0);
                sum += ml.y * f;
                v[0] += q.x * f, v[1] += q.y * f, v[2] += q.z * f, v[3] += q.w * f;
            }
            if (whole) {
                finish(s, row, d0, v, top, sum);
            } else {
                *(float4 *)(piece + row * D + d0) = make_float4(v[0], v[1], v[2], v[3]);
                if (d0 == 0) ((float2 *)(piece + kAttnPieceRows * D))[row] = make_float2(top, sum);
            }
        }
    }
    // the one that this block's run starts in the middle of, and the one it ends in the middle of: the blocks that
    // hold it count their arrivals, and the last one joins all pieces, in order
    if (sh.side[0].end == 0 && sh.side[1].end == 0) return;
    __syncthreads();
    if (threadIdx.x < 2) {
        const int side = threadIdx.x;
        bool final_one = false;
        __threadfence();                                    // for the block's writes, which the barrier orders before it
        if (sh.side[side].end != 0) {
            int *ticket = a.tickets + sh.first[side];
            final_one = atomicAdd(ticket, 1) == sh.last[side] - sh.first[side];
            if (final_one) *ticket = 0;
        }
        __threadfence();                                    // and for the reads of the block's threads after the next one
        sh.note[side] = final_one;
    }
    __syncthreads();
    for (int side = 0; side < 2; ++side) {
        if (!sh.note[side]) continue;
        const Rec s = sh.side[side];
        const int i0 = sh.first[side], i1 = sh.last[side];
        auto piece_of = [&](int p) { return a.pieces + ((int64_t)p * 2 + (p == i0)) * attn_piece_floats(D); };
        // A warp's rows at once (one after the other: 41.0 in place of 35.3 us for 32 sequences, 16 queries a group,
        // head_dim 64): a lane looks after a piece's weight, then after 4 of the row's elements.
        constexpr int RW = HT / kAttnWarps, AHEAD = 16 / RW;     // pieces asked for before their weights are known
        const int n_rows = rows_of(s);
        float top[RW], sum[RW], v[RW][4];
#pragma unroll
        for (int i = 0; i < RW; ++i) {
            top[i] = -INFINITY, sum[i] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = 0.f;
        }
        for (int from = i0; from <= i1; from += 32) {
            const int here = min(32, i1 + 1 - from);
            auto values = [&](int i, int p) {
                const int row = warp + kAttnWarps * i;
                return lane < D / 4 && p < here && row < n_rows
                           ? __ldcg((const float4 *)(piece_of(from + p) + row * D) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
            };
            float2 ml[RW];
            float4 q[RW][AHEAD];
#pragma unroll
            for (int i = 0; i < RW; ++i) {
                ml[i] = make_float2(-INFINITY, 0.f);
                if (lane < here && warp + kAttnWarps * i < n_rows)
                    ml[i] = __ldcg((const float2 *)(piece_of(from + lane) + kAttnPieceRows * D) + warp + kAttnWarps * i);
#pragma unroll
                for (int p = 0; p < AHEAD; ++p) q[i][p] = values(i, p);
            }
            float f[RW];
#pragma unroll
            for (int i = 0; i < RW; ++i) {
                const float up = fmaxf(top[i], warp_max(ml[i].x)), was = top[i] == -INFINITY ? 0.f : ex2(top[i] - up);
                f[i] = ml[i].x == -INFINITY ? 0.f : ex2(ml[i].x - up);
                sum[i] = sum[i] * was + warp_sum(ml[i].y * f[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] *= was;
                top[i] = up;
            }
            for (int p0 = 0; p0 < here; p0 += AHEAD) {
#pragma unroll
                for (int i = 0; i < RW; ++i)
#pragma unroll
                    for (int p = 0; p < AHEAD; ++p) {
                        const float fp = __shfl_sync(0xffffffffu, f[i], p0 + p);   // 0 past the last piece
                        if (p0 + p < here) {
                            v[i][0] += q[i][p].x * fp, v[i][1] += q[i][p].y * fp;
                            v[i][2] += q[i][p].z * fp, v[i][3] += q[i][p].w * fp;
                        }
                        q[i][p] = values(i, p0 + AHEAD + p);
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < RW; ++i)
            if (lane < D / 4 && warp + kAttnWarps * i < n_rows) finish(s, warp + kAttnWarps * i, 4 * lane, v[i], top[i], sum[i]);
    }
}

// The kernels of a format.  A group of more than 8 queries takes 16 a tile where its terms are few, and tiles of 8
// (each with its own pass over the keys) where they are many: with 16 a tile the terms of fp32 do not fit the
// registers.  16 sequences of 1000 to 4000 tokens, 16 queries a group, head_dim 128, fp32: 51 us in tiles of 8, 64 in
// tiles of 16; 12 queries, bf16, 32 sequences: 93 and 64 (an earlier form of the loop; 59 now).  16 queries, 32
// sequences of 1000 to 4000, head_dim 64: bf16 36 us, int8 37, e4m3 34.
enum AttnKind { ATTN_STACK, ATTN_STACK_EXACT, ATTN_PLAIN };
inline AttnKind attn_kind(int group, bool exact) {
    return exact ? ATTN_STACK_EXACT : group <= 8 ? ATTN_STACK : ATTN_PLAIN;
}

// Launches, and kernel limits of the current device; one translation unit per format.
cudaError_t launch_attention_bf16(int d, const AttnArg &a, AttnKind kind, int sms, cudaStream_t st);
cudaError_t launch_attention_int8(int d, const AttnArg &a, AttnKind kind, int sms, cudaStream_t st);
cudaError_t launch_attention_e4m3(int d, const AttnArg &a, AttnKind kind, int sms, cudaStream_t st);
cudaError_t launch_attention_e2m1(int d, const AttnArg &a, AttnKind kind, int sms, cudaStream_t st);
cudaError_t setup_attention_bf16();
cudaError_t setup_attention_int8();
cudaError_t setup_attention_e4m3();
cudaError_t setup_attention_e2m1();

template <int FMT, int D, bool STACK, bool EXACT>
cudaError_t launch_attention(const AttnArg &a, int sms, cudaStream_t st) {
    return launch_kernel(paged_attention_kernel<FMT, D, STACK, EXACT>, dim3(AttnShape<FMT, D, STACK>::kBlocks * sms), kAttnThreads,
                         AttnShape<FMT, D, STACK>::kSmem, st, 1, true, a);
}
template <int FMT, int D, bool STACK, bool EXACT>
cudaError_t limit_attention() {
    return cudaFuncSetAttribute(paged_attention_kernel<FMT, D, STACK, EXACT>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, AttnShape<FMT, D, STACK>::kSmem);
}

}  // namespace wici
