// Bounds of a cache's pages and the pages that a query's cheap score selects (include/wici_ops.h).
//
// Bounds.  bounds_kernel keeps, of each page and KV head, the largest and the smallest key element by element, as int8
// codes under one fp32 scale: (2 d + 4) bytes where the page's keys have 32 d (bf16).
//
// Scores.  sum_d max(q_d hi_d, q_d lo_d) is the largest q.k that keys between lo and hi can have.  q enters as whole
// numbers of at most 1023 (11 bits: fp16 holds them), the positive ones against hi and the negative ones against lo, so a
// score is a dot product of whole numbers whose sums stay below 2^24: mma.m16n8k16 gives it exactly, in any order, and the
// selection does not depend on how sums are split.  16 pages are the rows, 8 queries of the group the columns.
// Select.  A cluster of blocks takes one sequence and KV head.  Its blocks score the pages and leave the scores, as
// integers that order as they do, in the first block's shared memory; that one finds the keep-th largest by
// counting into bins, and writes the pages from it on in order, of equal ones the first.
// Measured (device time; 8 KV heads of 128, 4 queries each): 528 pages, 64 kept 7.6 us; 4 sequences of 6250 to 8192 pages,
// 256 kept 23.7 us, 2.5 TB/s of bounds; 32 sequences of 125 to 2048 pages, 128 kept 33.5 us.  What bounds it is latency: of
// the 23.7 us 9 pass before scores and between them (lengths, page numbers, rows; a tile's chain from its rows to its
// keys), 7 while copies are asked for, and 7 are the search and the lists of 32 blocks, in passes of one block each.  From
// L2 it is as fast.  Where a few scores lie far above the others, which then share a bin, the three take 2.4, 5.7 and 7 us
// more.  Bounds of 4096 pages: e4m3 19.7 us, 3.9 TB/s, bf16 23.8 us, 6.5 TB/s, e2m1 24 us, where a lane takes 2 bytes of a
// row and its block's scale, 16 times; of 64 pages 1.7 to 2.0 us.
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

// ------------------------------------------------------------------ bounds ----
struct BoundsArg {
    CacheArg cache;
    uint8_t *bounds;
    int64_t bounds_stride;
    const int32_t *last;
    int32_t *status;
    int64_t items;                    // entries of `last` times KV heads
};

constexpr int kBoundsThreads = 128;

// E values of a key row from element e0 on, as they stand, and as fp32 (the token's scale left out)
template <int FMT, int D, int E>
struct KeyPart {
    uint32_t w[FMT == WICI_KV_BF16 ? E / 2 : 1], each;
    __device__ __forceinline__ void load(const uint8_t *block, int row, int e0) {
        const uint8_t *p = block + row * kv_row_bytes(FMT, D) + (FMT == WICI_KV_BF16 ? 2 * e0 : FMT == WICI_KV_E2M1 ? e0 / 2 : e0);
        if (FMT == WICI_KV_BF16 && E == 4) {
            const uint2 v = *(const uint2 *)p;
            w[0] = v.x, w[E / 2 - 1] = v.y;
        } else if (FMT == WICI_KV_E2M1) {
            w[0] = E == 4 ? *(const uint16_t *)p : *p;
            each = block[kKvPage * (D / 2) + row * (D / 16) + e0 / 16];
        } else {
            w[0] = FMT == WICI_KV_BF16 || E == 4 ? *(const uint32_t *)p : *(const uint16_t *)p;
        }
    }
    __device__ __forceinline__ void values(float *x) const {
        if (FMT == WICI_KV_BF16) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) x[2 * i] = bf16lo(w[i]), x[2 * i + 1] = bf16hi(w[i]);
            return;
        }
        uint32_t h[4];
        if (FMT == WICI_KV_E2M1) decode_e2m1(w[0], h);
        else decode4<FMT>(w[0], h[0], h[1]);
        const float b = FMT == WICI_KV_E2M1 ? e4m3_value(each) : 1.f;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const float2 f = __half22float2(*(const __half2 *)&h[i]);
            x[2 * i] = FMT == WICI_KV_E2M1 ? f.x * b : f.x, x[2 * i + 1] = FMT == WICI_KV_E2M1 ? f.y * b : f.y;
        }
    }
};
// the largest and the smallest of three, NaN where one is
__device__ __forceinline__ float max_of(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float min_of(float a, float b, float c) {
    float d;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// A warp takes one page of one KV head, a lane E elements of all its rows, which it asks for at once and keeps as they
// stand: few registers, many warps.
template <int FMT, int D>
__global__ void __launch_bounds__(kBoundsThreads) bounds_kernel(const __grid_constant__ BoundsArg a) {
    constexpr int E = D / 32;
    griddep_launch_dependents();
    griddep_wait();
    const int64_t item = (int64_t)blockIdx.x * (kBoundsThreads / 32) + threadIdx.x / 32;
    if (item >= a.items) return;
    const int lane = threadIdx.x & 31, kv = a.cache.kv_heads, head = (int)((uint32_t)item % (uint32_t)kv);   // items <= 2^31
    const int last = a.last[(uint32_t)item / (uint32_t)kv];
    if (last < 0) return;
    const int page = last / kKvPage, rows = last % kKvPage + 1;
    if (page >= a.cache.n_pages) {
        if (lane == 0 && a.status) atomicOr(a.status, WICI_BAD_SLOT);
        return;
    }
    const uint8_t *block = a.cache.data + page * a.cache.page_stride + (int64_t)head * kv_block_bytes(FMT, D);
    KeyPart<FMT, D, E> part[kKvPage];
#pragma unroll
    for (int r = 0; r < kKvPage; ++r) part[r].load(block, r < rows ? r : 0, lane * E);   // past the last row: row 0 again
    float scale = 1.f;
    if (FMT != WICI_KV_BF16) scale = ((const float *)(block + kv_scales_at(FMT, D)))[lane < rows ? lane : 0];
    float hi[E], lo[E];               // NaN where one of the values is
    auto row = [&](int r, float *v) {
        part[r].values(v);
        if (FMT == WICI_KV_BF16) return;
        const float s = __shfl_sync(0xffffffffu, scale, r);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] *= s;
    };
    row(0, hi);
#pragma unroll
    for (int j = 0; j < E; ++j) lo[j] = hi[j];
#pragma unroll
    for (int r = 1; r < kKvPage; r += 2) {
        float u[E], v[E];
        row(r, u);
        row(r + 1 < kKvPage ? r + 1 : r, v);
#pragma unroll
        for (int j = 0; j < E; ++j) hi[j] = max_of(hi[j], u[j], v[j]), lo[j] = min_of(lo[j], u[j], v[j]);
    }
    uint32_t most = 0;                // of the magnitudes' bits: an infinity or NaN is the largest
#pragma unroll
    for (int j = 0; j < E; ++j)
        most = max(most, max(__float_as_uint(hi[j]) & 0x7FFFFFFFu, __float_as_uint(lo[j]) & 0x7FFFFFFFu));
    most = __reduce_max_sync(0xffffffffu, most);
    const bool finite = most < kInfBits;
    const float s = finite ? __fmul_rn(__uint_as_float(most), 1.f / 127.f) : __uint_as_float(0x7FC00000u);
    const bool some = finite && s >= 0x1p-126f;
    int8_t code[2][E];
    const float per = some ? 1.f / s : 0.f;
    auto whole = [&](float v) {       // the quotient v / s, right to its last bit, to the nearest whole number
        const float y = v * per;
        return (int8_t)__float2int_rn(fmaf(fmaf(-y, s, v), per, y));
    };
#pragma unroll
    for (int j = 0; j < E; ++j) code[0][j] = some ? whole(hi[j]) : (int8_t)0, code[1][j] = some ? whole(lo[j]) : (int8_t)0;
    uint8_t *record = a.bounds + page * a.bounds_stride;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint8_t *to = record + (head * 2 + i) * D + lane * E;
        if (E == 4) *(uint32_t *)to = *(const uint32_t *)code[i];
        else *(uint16_t *)to = *(const uint16_t *)code[i];
    }
    if (lane == 0) ((float *)(record + kv * 2 * D))[head] = finite ? some ? s : 0.f : s;
}

// ------------------------------------------------------------------ select ----
struct SelectArg {
    HeadsArg q;
    const uint8_t *bounds;
    int64_t bounds_stride;
    const int32_t *pages, *lengths;
    int32_t *out_pages, *out_lengths, *out_blocks, *status;
    int kv_heads, group, n_pages, max_pages, keep, first, recent, q_dtype;
    int cluster;
};

constexpr int kMaxSelectPages = 1 << 14;   // of a sequence: their scores stand in shared memory
constexpr int kMaxKeep = 1 << 12;          // and the selected ones
constexpr uint32_t kListed = 256;          // keys that are compared one with another, rather than counted
constexpr int kMaxSelectGroup = 64;        // query heads of a KV head: so do they
constexpr float kLevels = 1023.f;          // of a query's whole numbers: 128 * 127 * 1023 < 2^24
constexpr int kBinBits = 11, kBins = 1 << kBinBits;
constexpr uint32_t kForced = 0xFFFFFFFFu;  // in the place of a score: above every one
constexpr uint32_t kFirst = 0xFF800000u;   // +infinity's

constexpr size_t select_smem(int d, int warps, int tile, int group, int max_pages, int keep) {
    return (size_t)warps * tile * 2 * d + (size_t)(group + 7) / 8 * (2 * d / 16 * 256 + 8 * 12) + ((size_t)max_pages + 31) / 32 * 128 + (size_t)keep * 2;
}

// Scores in the order of unsigned integers; NaN, which no page should have, stands with +infinity
__device__ __forceinline__ uint32_t order_of(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);
    if (s != s) return kFirst;
    return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
constexpr size_t kSelectSmem = 217 * 1024;   // at most, beside what the kernel has of its own
constexpr size_t kSelectOwn = kBins * 4 + 1536;   // that, and what every block of an SM has besides
constexpr size_t kSmSmem = 228 * 1024;            // of an SM
constexpr int kFewPages = 2048;                   // four blocks of 4 warps fit with these, and few heads a group
static_assert(select_smem(128, 16, 16, kMaxSelectGroup, kMaxSelectPages, kMaxKeep) <= kSelectSmem, "the largest call");
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float score_of(uint32_t order) {
    return __uint_as_float(order >> 31 ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ void mma_f16(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint2 b) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ void store_to_first(uint32_t addr, uint32_t v) {
    asm volatile("{\n\t.reg .u32 ra;\n\tmapa.shared::cluster.u32 ra, %0, 0;\n\tst.shared::cluster.u32 [ra], %1;\n\t}" ::"r"(addr), "r"(v)
                 : "memory");
}

template <int D, int kSelectThreads, int kTile>
__global__ void __launch_bounds__(kSelectThreads, 512 / kSelectThreads) select_kernel(const __grid_constant__ SelectArg a) {
    constexpr int kSelectWarps = kSelectThreads / 32, GROUPS = kTile / 8;   // of 8 pages of a tile
    constexpr int STEPS = 2 * D / 16, ROW = 2 * D;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ uint32_t part[2][kSelectWarps], bins[kBins], ends[2][8 * kSelectWarps], listed;
    const int tiles = (a.group + 7) / 8;
    const uint32_t rows_at = smem_u32(smem) + threadIdx.x / 32 * kTile * ROW;   // this warp's: [page of a tile]
    __half *qs = (__half *)(smem + kSelectWarps * kTile * ROW);                 // [tile][step][lane][4]: B fragments
    float *most = (float *)((uint8_t *)qs + tiles * STEPS * 256); // [tile * 8]: each query's largest magnitude
    float2 *bias = (float2 *)(most + tiles * 8);                  // [tile * 8]: 128 times the sums of its whole numbers
    uint32_t *keys = (uint32_t *)(bias + tiles * 8);              // [page], of the first block
    uint16_t *chosen = (uint16_t *)(keys + (a.max_pages + 31) / 32 * 32);   // [keep]
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rank = blockIdx.x % a.cluster, h = blockIdx.x / a.cluster, b = blockIdx.y;
    // Every block of a cluster comes to each barrier, whatever it reads
    if (a.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    griddep_launch_dependents();
    griddep_wait();
    const int n = a.lengths[b];
    const bool bad = n > (int64_t)a.max_pages * kKvPage;
    const int count = bad || n <= 0 ? 0 : (n + kKvPage - 1) / kKvPage;
    const bool choose = count > a.keep;
    const int32_t *table = a.pages + (int64_t)b * a.max_pages;
    // A tile is kTile pages, lane l looks after page l (l % 16).  Tiles come through cp.async, the next one asked for when
    // this one has been read: what waits for it is hidden by other warps, and a second one under way was no faster.  (Loads
    // to registers wait in L1, which the attention's shared memory leaves small: 46 in place of 30 us beside it.)
    const int step = kSelectWarps * a.cluster, first_tile = rank * kSelectWarps + warp;
    const uint64_t policy = l2_evict_first();
    const uint32_t stride = (uint32_t)a.bounds_stride;            // below 2^31
    auto page_of = [&](int tile) {
        const int at = tile * kTile + lane % kTile;
        return choose && at < count ? table[at] : 0;
    };
    constexpr int CHUNKS = ROW / 16, ROUNDS = kTile * CHUNKS / 32;   // of a row; rounds of the warp for a tile
    const uint8_t *const of_lane = a.bounds + h * ROW + lane % CHUNKS * 16;
    const uint8_t *const of_scale = a.bounds + a.kv_heads * ROW + 4 * h;
    // chunks of odd rows with their halves of 128 bytes exchanged: lanes that read 64 bytes of two rows meet all banks
    const uint32_t copy_to = rows_at + lane / CHUNKS * ROW + ((lane % CHUNKS ^ (lane / CHUNKS & 1) << 2) << 4);
    struct Asked {                                                // of the lane's page
        float scale;                                              // not looked at before it is needed: it is still on its way
        bool there;
    };
    auto ask = [&](int tile, int page) {
        if (!choose || tile * kTile >= count) return Asked{0.f, false};
        const bool there = (uint32_t)page < (uint32_t)a.n_pages;
        if (!there && a.status) atomicOr(a.status, WICI_BAD_PAGE);
        const int p = there ? page : 0;                           // (of page 0, not used)
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int of = __shfl_sync(0xffffffffu, p, i * (32 / CHUNKS) + lane / CHUNKS);
            cp_async16(copy_to + i * 512, of_lane + (uint64_t)(uint32_t)of * stride, policy);
        }
        return Asked{*(const float *)(of_scale + (uint64_t)(uint32_t)p * stride), there};
    };
    int next_page = page_of(first_tile);
    Asked asked = ask(first_tile, next_page);
    next_page = page_of(first_tile + step);

    if (choose) {
        for (int i = warp; i < tiles * 8; i += kSelectWarps) {    // one query a warp
            float x[D / 32];
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                x[j] = 0.f;
                if (i < a.group) {
                    const int64_t e = lane + 32 * j;
                    const int head = h * a.group + i;
                    x[j] = a.q_dtype == WICI_F32 ? a.q.row<float>(b, head)[e]
                           : a.q_dtype == WICI_F16 ? __half2float(a.q.row<__half>(b, head)[e])
                                                   : __bfloat162float(a.q.row<__nv_bfloat16>(b, head)[e]);
                }
                top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
            }
            top = __reduce_max_sync(0xffffffffu, top);
            const bool some = top < kInfBits && __uint_as_float(top) >= 0x1p-100f;
            const float per = some ? __fmul_rn(__frcp_rn(__uint_as_float(top)), kLevels) : 0.f;
            float sums[2] = {0.f, 0.f};                           // over elements of even and of odd words
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                const float w = some ? rintf(__fmul_rn(x[j], per)) : 0.f;
#pragma unroll
                for (int end = 0; end < 2; ++end) {               // against the largest keys, the smallest
                    const int e = end * D + lane + 32 * j;        // byte of a record's row: chunk e / 16 is lane t's
                    const int at = e / 64 * 4 + e % 16 / 4, to = i % 8 * 4 + e / 16 % 4;
                    qs[((i / 8 * STEPS + at) * 32 + to) * 4 + e % 4] = __float2half_rn(end ? fminf(w, 0.f) : fmaxf(w, 0.f));
                }
                sums[lane >> 2 & 1] += w;
            }
            sums[0] = warp_sum(sums[0]), sums[1] = warp_sum(sums[1]);
            if (lane == 0) most[i] = some ? __uint_as_float(top) : 0.f, bias[i] = make_float2(128.f * sums[0], 128.f * sums[1]);
        }
    }
    __syncthreads();
    if (a.cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // the first block runs

    uint32_t hi = 0, lo = 0xFFFFFFFFu;                            // of this lane's scores that are not forced
    if (choose) {
        const uint32_t keys_at = smem_u32(keys);
        const uint32_t row = rows_at + g * ROW + 16 * t, even = (g & 1) << 6;
        for (int tile = first_tile; tile * kTile < count; tile += step) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
            float best[GROUPS];                                   // of pages g + 8 r
#pragma unroll
            for (int r = 0; r < GROUPS; ++r) best[r] = -INFINITY;
            for (int q = 0; q < tiles; ++q) {
                // codes + 128 as they are are fp16's smallest numbers, 2^-24 each: sums of 64 products with whole numbers up
                // to 1023 stay below 2^24 of them, and 128 times the whole numbers' sum is taken off after
                float c[GROUPS / 2][2][4] = {};                   // [16 pages][sums side by side]
                const uint2 *frag = (const uint2 *)qs + q * STEPS * 32 + lane;
#pragma unroll
                for (int i = 0; i < STEPS / 4; ++i) {
                    const uint32_t at = row + (i & 1 ? even ^ 64 : even) + i / 2 * 128;
                    uint32_t w[GROUPS][4];
#pragma unroll
                    for (int r = 0; r < GROUPS; ++r) {
                        const uint4 v = lds128(at + 8 * r * ROW);
                        w[r][0] = v.x ^ 0x80808080u, w[r][1] = v.y ^ 0x80808080u, w[r][2] = v.z ^ 0x80808080u, w[r][3] = v.w ^ 0x80808080u;
                    }
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const uint2 f = frag[(4 * i + s) * 32];
#pragma unroll
                        for (int k = 0; k < GROUPS / 2; ++k)
                            mma_f16(c[k][s & 1], __byte_perm(w[2 * k][s], 0, 0x4140), __byte_perm(w[2 * k + 1][s], 0, 0x4140),
                                    __byte_perm(w[2 * k][s], 0, 0x4342), __byte_perm(w[2 * k + 1][s], 0, 0x4342), f);
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int head = q * 8 + 2 * t + j;
                    const float m = most[head];
                    const float2 off = bias[head];
#pragma unroll
                    for (int r = 0; r < GROUPS; ++r) {
                        const int x = 2 * (r & 1) + j;
                        const float dot = fmaf(c[r >> 1][0][x], 0x1p24f, -off.x) + fmaf(c[r >> 1][1][x], 0x1p24f, -off.y);
                        best[r] = fmaxf(best[r], head < a.group ? __fmul_rn(dot, m) : -INFINITY);
                    }
                }
            }
            const float of_page = asked.there ? asked.scale : INFINITY;
            __syncwarp();                                         // the rows have been read
            asked = ask(tile + step, next_page);
            next_page = page_of(tile + 2 * step);
#pragma unroll
            for (int r = 0; r < GROUPS; ++r) {
                best[r] = fmaxf(best[r], __shfl_xor_sync(0xffffffffu, best[r], 1));
                best[r] = fmaxf(best[r], __shfl_xor_sync(0xffffffffu, best[r], 2));
            }
            // lane (g, t) has page g + 8 t now (of 16 pages, half of the lanes)
            const int of_t = t & (GROUPS - 1);
            float mine = best[0];
#pragma unroll
            for (int r = 1; r < GROUPS; ++r) mine = of_t == r ? best[r] : mine;
            const float scale = __shfl_sync(0xffffffffu, of_page, g + 8 * of_t);
            const int i = tile * kTile + g + 8 * of_t;
            uint32_t key = kFirst;                                // a key that is not finite, a page that is not there
            if (scale == 0.f) key = order_of(0.f);
            else if (fabsf(scale) < INFINITY) key = order_of(__fmul_rn(mine, scale));
            if (i < a.first || i >= count - a.recent) key = kForced;
            else hi = max(hi, key), lo = min(lo, key);
            if (i < count) {
                if (a.cluster > 1) store_to_first(keys_at + 4 * i, key);
                else keys[i] = key;
            }
        }
        hi = __reduce_max_sync(0xffffffffu, hi);
        lo = __reduce_min_sync(0xffffffffu, lo);
        if (lane == 0) {
            const int at = rank * kSelectWarps + warp;
            if (a.cluster > 1) store_to_first(smem_u32(&ends[0][at]), hi), store_to_first(smem_u32(&ends[1][at]), lo);
            else ends[0][at] = hi, ends[1][at] = lo;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (rank == 0)
        for (int i = threadIdx.x; i < kBins; i += kSelectThreads) bins[i] = 0;
    if (threadIdx.x == 0) listed = 0;
    if (a.cluster > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank != 0) return;
    } else {
        __syncthreads();
    }

    // ---- the first block: the keep-th largest key, and the pages from it on ----
    int32_t *pages = a.out_pages + ((int64_t)b * a.kv_heads + h) * a.keep;
    int32_t *blocks = a.out_blocks ? a.out_blocks + ((int64_t)b * a.kv_heads + h) * a.keep : nullptr;
    if (h == 0 && threadIdx.x == 0) {
        // what is bad stays bad: a length past the selected pages
        a.out_lengths[b] = bad ? a.keep * kKvPage + 1 : choose ? (a.keep - 1) * kKvPage + (n - 1) % kKvPage + 1 : max(n, 0);
        if (bad && a.status) atomicOr(a.status, WICI_BAD_LENGTH);
    }
    if (!choose) {
        for (int i = threadIdx.x; i < a.keep; i += kSelectThreads) {
            const int page = i < count ? table[i] : -1;
            pages[i] = page;
            if (blocks) blocks[i] = i < count ? i : -1;
            if (h == 0 && i < count && (uint32_t)page >= (uint32_t)a.n_pages && a.status) atomicOr(a.status, WICI_BAD_PAGE);
        }
        return;
    }
    uint32_t limit = kForced;
    if (a.first + a.recent < a.keep) {
        // over the keys that are not forced and that `in` takes: a count for each value of `bin` (bins are 0 before), and
        // then the bin that has the keep-th largest of all, where `above` keys are known to be larger
        uint32_t above = a.first + a.recent;
        auto narrow = [&](auto in, auto bin) {
#pragma unroll 4
            for (int i = threadIdx.x; i < count; i += kSelectThreads) {
                const uint32_t k = keys[i];
                if (k != kForced && in(k)) atomicAdd(&bins[bin(k)], 1u);
            }
            __syncthreads();
            constexpr int kEach = kBins / kSelectThreads;         // bins of a thread, the highest first
            const int top = kBins - 1 - kEach * threadIdx.x;
            uint32_t mine = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) mine += bins[top - i];
            uint32_t upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            if (lane == 31) part[0][warp] = upto;
            __syncthreads();
            for (int w = 0; w < warp; ++w) upto += part[0][w];
            uint32_t before = above + upto - mine;
            if (before < (uint32_t)a.keep && before + mine >= (uint32_t)a.keep) {
                int at = top;
                while (before + bins[at] < (uint32_t)a.keep) before += bins[at--];
                part[1][0] = at;
                part[1][1] = before;
                part[1][2] = bins[at];
            }
            __syncthreads();
            above = part[1][1];
            return part[1][0];
        };
        hi = 0, lo = 0xFFFFFFFFu;                                 // the largest and the smallest of them
        for (int w = lane; w < step; w += 32) hi = max(hi, ends[0][w]), lo = min(lo, ends[1][w]);
        hi = __reduce_max_sync(0xffffffffu, hi);
        lo = __reduce_min_sync(0xffffffffu, lo);
        limit = hi;
        if (hi != lo) {
            // Bins of equal width first: bits of scores, of like size as they are, would fall into few bins, whose counting
            // takes turns.  The bin of a score grows with it, whatever is rounded.  (Not where the width is no number.)
            const float least = score_of(lo), per = (kBins - 1) / (score_of(hi) - least);
            const bool even = per > 0.f && per < INFINITY;
            auto bin = [=](uint32_t k) { return even ? min(kBins - 1, max(0, (int)((score_of(k) - least) * per))) : 0; };
            const int found = even ? (int)narrow([](uint32_t) { return true; }, bin) : 0;
            const uint32_t in_bin = even ? part[1][2] : 0xFFFFFFFFu;
            __syncthreads();
            if (in_bin <= kListed) {
                // few keys: each is compared with the others
                uint32_t *list = bins;
#pragma unroll 4
                for (int i = threadIdx.x; i < count; i += kSelectThreads) {
                    const uint32_t k = keys[i];
                    if (k != kForced && bin(k) == found) list[atomicAdd(&listed, 1u) & (kListed - 1)] = k;
                }
                __syncthreads();
                for (uint32_t i = threadIdx.x; i < in_bin; i += kSelectThreads) {
                    const uint32_t k = list[i];
                    uint32_t larger = above, equal = 0;
                    for (uint32_t j = 0; j < in_bin; ++j) larger += list[j] > k, equal += list[j] == k;
                    if (larger < (uint32_t)a.keep && larger + equal >= (uint32_t)a.keep) part[0][0] = k;
                }
                __syncthreads();
                limit = part[0][0];
            } else {
                // many: of the keys in the bin, kBinBits of their bits at a time from the first that differ
                hi = 0, lo = 0xFFFFFFFFu;
                for (int i = threadIdx.x; i < count; i += kSelectThreads) {
                    const uint32_t k = keys[i];
                    if (k != kForced && bin(k) == found) hi = max(hi, k), lo = min(lo, k);
                }
                hi = __reduce_max_sync(0xffffffffu, hi);
                lo = __reduce_min_sync(0xffffffffu, lo);
                if (lane == 0) part[0][warp] = hi, part[1][warp] = lo;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kSelectWarps; ++w) hi = max(hi, part[0][w]), lo = min(lo, part[1][w]);
                int open = hi == lo ? 0 : 32 - __clz(hi ^ lo);
                const uint32_t most_key = hi, least_key = lo;
                limit = open == 32 ? 0u : hi >> open << open;
                while (open > 0) {
                    __syncthreads();                              // `part` and `bins` have been read
                    for (int i = threadIdx.x; i < kBins; i += kSelectThreads) bins[i] = 0;
                    __syncthreads();
                    const int low = open > kBinBits ? open - kBinBits : 0;
                    const uint32_t mask = (1u << (open - low)) - 1, prefix = limit;
                    limit |= narrow([=](uint32_t k) { return k >= least_key && k <= most_key && (open == 32 || (k ^ prefix) >> open == 0); },
                                    [=](uint32_t k) { return (k >> low) & mask; }) << low;
                    open = low;
                }
            }
        }
    }
    // a warp's share of the pages, in order: those above the limit, and as many of those at it as there is room for
    const int share = ((count + kSelectWarps - 1) / kSelectWarps + 31) & ~31, from = warp * share, to = min(count, from + share);
    uint32_t over = 0, at = 0;
#pragma unroll 4
    for (int i = from + lane; i < to; i += 32) over += keys[i] > limit, at += keys[i] == limit;
    over = __reduce_add_sync(0xffffffffu, over);
    at = __reduce_add_sync(0xffffffffu, at);
    __syncthreads();                                              // what was left in `part` has been read
    if (lane == 0) part[0][warp] = over, part[1][warp] = at;
    __syncthreads();
    uint32_t all_over = 0;
#pragma unroll
    for (int w = 0; w < kSelectWarps; ++w) all_over += part[0][w];
    uint32_t room = a.keep > (int)all_over ? a.keep - all_over : 0, place = 0;
    for (int w = 0; w < warp; ++w) {
        const uint32_t taken = min(room, part[1][w]);
        place += part[0][w] + taken;
        room -= taken;
    }
    const uint32_t below = (1u << lane) - 1;
    for (int i0 = from; i0 < to; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t k = i < to ? keys[i] : 0u;
        const bool is_over = i < to && k > limit, is_at = i < to && k == limit;
        const uint32_t m_at = __ballot_sync(0xffffffffu, is_at);
        const bool taken = is_over || (is_at && (uint32_t)__popc(m_at & below) < room);
        const uint32_t m = __ballot_sync(0xffffffffu, taken);
        const uint32_t p = place + __popc(m & below);
        if (taken && p < (uint32_t)a.keep) chosen[p] = (uint16_t)i;
        place += __popc(m);
        room -= min(room, (uint32_t)__popc(m_at));
    }
    __syncthreads();
    for (int p = threadIdx.x; p < a.keep; p += kSelectThreads) {
        const int i = min((int)chosen[p], count - 1);
        pages[p] = table[i];
        if (blocks) blocks[p] = i;
    }
}

template <int D>
cudaError_t limit_select(int most) {
    cudaError_t e = cudaFuncSetAttribute(select_kernel<D, 128, 32>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(select_kernel<D, 512, 16>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(select_kernel<D, 512, 32>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return e;
}
template <int D>
cudaError_t launch_select(int threads, int tile, dim3 grid, size_t smem, cudaStream_t st, const SelectArg &a) {
    if (threads == 128) return launch_kernel(select_kernel<D, 128, 32>, grid, 128, smem, st, a.cluster, true, a);
    return tile == 32 ? launch_kernel(select_kernel<D, 512, 32>, grid, 512, smem, st, a.cluster, true, a)
                      : launch_kernel(select_kernel<D, 512, 16>, grid, 512, smem, st, a.cluster, true, a);
}

// the most blocks of a cluster that the current device has room for, with the most shared memory: 8 unless it is a part of one
cudaError_t resident_cluster(int *most) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.blockDim = dim3(512);
    cfg.dynamicSmemBytes = kSelectSmem;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    for (*most = 8; *most > 1; *most /= 2) {
        attr.val.clusterDim.x = *most;
        cfg.gridDim = dim3(*most);
        int n = 0;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, select_kernel<128, 512, 32>, &cfg);
        if (e != cudaSuccess) return e;
        if (n > 0) break;
    }
    return cudaSuccess;
}

struct Device {
    int sms, cluster;
};
DeviceTable<Device> g_devices;

int device_of(Device *d) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
        e = g_devices.get(dev, d, [dev](Device *x) {
            constexpr int kMost = kSelectSmem;
            cudaError_t e1 = limit_select<64>(kMost);
            if (e1 == cudaSuccess) e1 = limit_select<128>(kMost);
            if (e1 == cudaSuccess) e1 = resident_cluster(&x->cluster);
            return e1 == cudaSuccess ? cudaDeviceGetAttribute(&x->sms, cudaDevAttrMultiProcessorCount, dev) : e1;
        });
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "select setup: %s", cudaGetErrorString(e));
}

const char *check_bounds(const wici_kv_bounds *b, const wici_kv_cache *c) {
    if (!b) return "null bounds";
    if (!b->data || ((uintptr_t)b->data & 15)) return "bounds data null or not 16-byte aligned";
    if (b->page_stride % 16 || b->page_stride < wici_kv_bounds_bytes(c->n_kv_heads, c->head_dim))
        return "bounds page_stride must be a multiple of 16 and at least a record";
    if (b->page_stride > INT32_MAX) return "bounds page_stride must be below 2^31";
    return nullptr;
}

bool overlap(const void *a, int64_t na, const void *b, int64_t nb) {
    return a && b && (uintptr_t)a < (uintptr_t)b + (size_t)nb && (uintptr_t)b < (uintptr_t)a + (size_t)na;
}
// whether n bytes at p meet one of `count` rows of `len` bytes, `stride` apart (what lies between them is not the rows')
bool meets(const void *p, int64_t n, const void *rows, int64_t count, int64_t stride, int64_t len) {
    if (!p || !overlap(p, n, rows, (count - 1) * stride + len)) return false;
    const int64_t at = (int64_t)((uintptr_t)p - (uintptr_t)rows);
    const int64_t i = at < len || stride == 0 ? 0 : (at - len) / stride + 1;   // the first row that ends behind p
    return i < count && i * stride < at + n;
}
bool meets(const void *p, int64_t n, const wici_heads *t, int64_t tokens, int d) {
    const int64_t e = dtype_bytes(t->dtype), token = t->token_stride * e, head = t->head_stride * e;
    if (!overlap(p, n, t->data, (tokens - 1) * token + (t->heads - 1) * head + d * e)) return false;
    for (int64_t i = 0; i < tokens; ++i)
        if (meets(p, n, (const uint8_t *)t->data + i * token, t->heads, head, d * e)) return true;
    return false;
}

template <int FMT>
cudaError_t launch_bounds(int d, const BoundsArg &a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.items + kBoundsThreads / 32 - 1) / (kBoundsThreads / 32)));
    return d == 64 ? launch_kernel(bounds_kernel<FMT, 64>, grid, kBoundsThreads, 0, st, 1, true, a)
                   : launch_kernel(bounds_kernel<FMT, 128>, grid, kBoundsThreads, 0, st, 1, true, a);
}

}  // namespace

extern "C" {

int64_t wici_kv_bounds_bytes(int32_t n_kv_heads, int32_t head_dim) {
    if ((head_dim != 64 && head_dim != 128) || n_kv_heads < 1) return 0;
    return ((int64_t)n_kv_heads * (2 * head_dim + 4) + 15) / 16 * 16;
}

int wici_kv_bounds_update(void *cuda_stream, const wici_kv_cache *cache, const wici_kv_bounds *bounds, const int32_t *last,
                          int64_t count, int32_t *status) {
    if (const char *m = check_cache(cache)) return fail(WICI_E_ARG, "bounds: %s", m);
    if (const char *m = check_bounds(bounds, cache)) return fail(WICI_E_ARG, "bounds: %s", m);
    if (count < 0 || count > kMaxPages) return fail(WICI_E_ARG, "bounds: count must be in [0, 2^27)");
    if (count == 0) return WICI_OK;
    if (!last || !words(last) || !words(status)) return fail(WICI_E_ARG, "bounds: last null, or last or status unaligned");
    BoundsArg a = {};
    a.cache = cache_arg(cache);
    a.bounds = (uint8_t *)bounds->data;
    a.bounds_stride = bounds->page_stride;
    a.status = status;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    const int64_t most = ((int64_t)1 << 31) / cache->n_kv_heads;    // of a launch: its blocks are below 2^30
    for (int64_t i = 0; i < count && e == cudaSuccess; i += most) {
        a.last = last + i;
        a.items = (count - i < most ? count - i : most) * cache->n_kv_heads;
        switch (cache->format) {
            case WICI_KV_BF16: e = launch_bounds<WICI_KV_BF16>(cache->head_dim, a, st); break;
            case WICI_KV_INT8: e = launch_bounds<WICI_KV_INT8>(cache->head_dim, a, st); break;
            case WICI_KV_E2M1: e = launch_bounds<WICI_KV_E2M1>(cache->head_dim, a, st); break;
            default: e = launch_bounds<WICI_KV_E4M3>(cache->head_dim, a, st); break;
        }
    }
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "bounds: %s", cudaGetErrorString(e));
}

int wici_kv_select(void *cuda_stream, const wici_kv_cache *cache, const wici_kv_bounds *bounds, const wici_select_shape *shape,
                   const int32_t *pages, const int32_t *lengths, const wici_heads *q, int32_t *out_pages,
                   int32_t *out_lengths, int32_t *out_blocks, int32_t *status) {
    if (const char *m = check_cache(cache)) return fail(WICI_E_ARG, "select: %s", m);
    if (const char *m = check_bounds(bounds, cache)) return fail(WICI_E_ARG, "select: %s", m);
    if (!shape) return fail(WICI_E_ARG, "select: null shape");
    if (shape->batch < 0 || shape->batch > 65535) return fail(WICI_E_ARG, "select: batch must be in [0, 65535]");
    if (shape->max_pages < 1 || shape->max_pages > kMaxSelectPages) return fail(WICI_E_ARG, "select: max_pages must be in [1, 16384]");
    if (shape->first < 0 || shape->recent < 1 || shape->keep < 1 || shape->keep > kMaxKeep ||
        shape->first > shape->keep || shape->recent > shape->keep - shape->first)
        return fail(WICI_E_ARG, "select: first >= 0, recent >= 1 and first + recent <= keep <= 4096 required");
    if (const char *m = check_heads(q, shape->batch, cache->head_dim, false)) return fail(WICI_E_ARG, "select q: %s", m);
    if (q->heads % cache->n_kv_heads || q->heads / cache->n_kv_heads > kMaxSelectGroup)
        return fail(WICI_E_ARG, "select: query heads must be a multiple of the cache's heads, at most 64 times as many");
    if (shape->batch == 0) return WICI_OK;
    if (!pages || !lengths || !out_pages || !out_lengths) return fail(WICI_E_ARG, "select: null pages or lengths");
    if (!words(pages) || !words(lengths) || !words(out_pages) || !words(out_lengths) || !words(out_blocks) || !words(status))
        return fail(WICI_E_ARG, "select: pages, lengths, blocks or status unaligned");
    const int64_t in = (int64_t)shape->batch * shape->max_pages * 4, list = (int64_t)shape->batch * cache->n_kv_heads * shape->keep * 4;
    const int64_t len = (int64_t)shape->batch * 4;
    const struct { const void *p; int64_t n; } outs[3] = {{out_pages, list}, {out_lengths, len}, {out_blocks, list}};
    for (int i = 0; i < 3; ++i) {
        bool shared = overlap(outs[i].p, outs[i].n, pages, in) || overlap(outs[i].p, outs[i].n, lengths, len) ||
                      overlap(outs[i].p, outs[i].n, status, 4) || meets(outs[i].p, outs[i].n, q, shape->batch, cache->head_dim) ||
                      meets(outs[i].p, outs[i].n, bounds->data, cache->n_pages, bounds->page_stride,
                            wici_kv_bounds_bytes(cache->n_kv_heads, cache->head_dim)) ||
                      meets(outs[i].p, outs[i].n, cache->data, cache->n_pages, cache->page_stride,
                            wici_kv_page_bytes(cache->format, cache->n_kv_heads, cache->head_dim));
        for (int j = 0; j < i; ++j) shared |= overlap(outs[i].p, outs[i].n, outs[j].p, outs[j].n);
        if (shared) return fail(WICI_E_ARG, "select: an output overlaps another tensor");
    }
    Device dev;
    if (int rc = device_of(&dev)) return rc;
    SelectArg a = {};
    a.q = heads_arg(q);
    a.bounds = (const uint8_t *)bounds->data;
    a.bounds_stride = bounds->page_stride;
    a.pages = pages;
    a.lengths = lengths;
    a.out_pages = out_pages;
    a.out_lengths = out_lengths;
    a.out_blocks = out_blocks;
    a.status = status;
    a.kv_heads = cache->n_kv_heads;
    a.group = q->heads / cache->n_kv_heads;
    a.n_pages = cache->n_pages;
    a.max_pages = shape->max_pages;
    a.keep = shape->keep;
    a.first = shape->first;
    a.recent = shape->recent;
    a.q_dtype = q->dtype;
    // Blocks of 16 warps where sequences and heads do not fill the SMs by themselves, of 4 where they do: 96 x 8 heads of up
    // to 250 pages 24 us (34 with 16), 32 x 8 of up to 2048 33.5 (34.5), but 4 x 8 of 8192 39 with 4 warps (24 with 16).
    // Blocks of a cluster: as many as there are SMs for (with twice as many 43 us in place of 26.7, in tiles of 16), and
    // pages for a tile a warp.
    const int64_t pairs = (int64_t)a.kv_heads * shape->batch;
    auto smem_of = [&](int warps, int tile) { return select_smem(cache->head_dim, warps, tile, a.group, a.max_pages, a.keep); };
    auto cluster_of = [&](int threads) {
        int c = 1;
        while (c < dev.cluster && 2 * c * pairs * threads <= (int64_t)512 * dev.sms && c * (threads / 32) * 16 < a.max_pages) c *= 2;
        return c;
    };
    int threads = pairs > dev.sms ? 128 : 512;
    if (threads == 128 && a.max_pages > kFewPages) {
        // Many pages: their scores leave an SM room for fewer blocks of 4 warps, and those take more waves.  A warp's share of
        // the pages in all waves, of 4 warps and of 16 (whose waves cost 1.4 times that: nothing runs beside a block's ends):
        // 20 x 8 heads of 8192 pages 110 us with 16 warps, 140 with 4; of 6000 84 and 74; 32 x 8 of 16384, 4096 kept, 237 and
        // 498; 64 x 8 of 4096 129 and 148; 96 x 8 of these 191 and 176.
        const int c = cluster_of(128), fit = (int)(kSmSmem / (smem_of(4, 32) + kSelectOwn));
        const int64_t room = (int64_t)(fit < 4 ? fit : 4) * dev.sms;
        const int64_t waves4 = (pairs * c + room - 1) / room, waves16 = (pairs + dev.sms - 1) / dev.sms;
        if (20 * waves4 > 7 * c * waves16) threads = 512;
    }
    const int warps = threads / 32;
    a.cluster = cluster_of(threads);
    // Tiles of 32 pages, which cost less a page (the 4 x 8 heads 23.7 us, 26.7 with 16), but of 16 where each warp has one of
    // these at most (528 pages 7.6 us, 9.6 with 32), and where 32 take more shared memory than there is.
    const int tile = threads == 128 || (a.cluster * warps * 16 < a.max_pages && smem_of(warps, 32) <= kSelectSmem) ? 32 : 16;
    const dim3 grid((unsigned)(a.cluster * a.kv_heads), (unsigned)shape->batch);
    const size_t smem = smem_of(warps, tile);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = cache->head_dim == 64 ? launch_select<64>(threads, tile, grid, smem, st, a)
                                                : launch_select<128>(threads, tile, grid, smem, st, a);
    return e == cudaSuccess ? WICI_OK : fail(WICI_E_CUDA, "select: %s", cudaGetErrorString(e));
}

}  // extern "C"
