// What the stand-alone operators of a batched decode step (include/wici_ops.h) share on the
// host: argument checks.  No CUDA needed, so that the checks can be tested by themselves.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/wici_ops.h"

namespace wici {

constexpr int kKvPage = 16;            // tokens of a page
constexpr int kMaxPages = (1 << 27) - 1;   // slots stay below 2^31
constexpr int kMaxHeads = 1 << 16;

inline int dtype_bytes(int dtype) { return dtype == WICI_F32 ? 4 : 2; }

// bytes of a token's elements in a [K or V][kv head] block of a page, and of the block: values, or codes (then e2m1's
// scales of 16 elements) and 16 fp32 scales
constexpr int kv_row_bytes(int format, int head_dim) {
    return format == WICI_KV_BF16 ? head_dim * 2 : format == WICI_KV_E2M1 ? head_dim / 2 : head_dim;
}
constexpr int kv_scales_at(int format, int head_dim) {    // of the fp32 scales in a block
    return kKvPage * (kv_row_bytes(format, head_dim) + (format == WICI_KV_E2M1 ? head_dim / 16 : 0));
}
constexpr int kv_block_bytes(int format, int head_dim) {
    return kv_scales_at(format, head_dim) + (format == WICI_KV_BF16 ? 0 : kKvPage * 4);
}
inline bool known_format(int f) {
    return f == WICI_KV_BF16 || f == WICI_KV_INT8 || f == WICI_KV_E4M3 || f == WICI_KV_E2M1;
}

inline const char *check_cache(const wici_kv_cache *c) {
    if (!c) return "null cache";
    if (!known_format(c->format)) return "cache format";
    if (c->head_dim != 64 && c->head_dim != 128) return "cache head_dim must be 64 or 128";
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return "cache n_kv_heads must be in [1, 1024]";
    if (c->n_pages < 1 || c->n_pages > kMaxPages) return "cache n_pages must be in [1, 2^27)";
    if (!c->data || ((uintptr_t)c->data & 15)) return "cache data null or not 16-byte aligned";
    if (c->page_stride % 16 || c->page_stride < 2 * (int64_t)c->n_kv_heads * kv_block_bytes(c->format, c->head_dim))
        return "cache page_stride must be a multiple of 16 and at least a page";
    if (c->page_stride > INT64_MAX / kMaxPages) return "cache page_stride";
    return nullptr;
}

// `tokens` x t->heads x d; out: a written tensor, whose elements have a place each
inline const char *check_heads(const wici_heads *t, int64_t tokens, int d, bool out) {
    if (!t) return "null tensor";
    if (t->dtype != WICI_BF16 && t->dtype != WICI_F16 && t->dtype != WICI_F32) return "element type";
    if (t->heads < 1 || t->heads > kMaxHeads) return "heads must be in [1, 65536]";
    if (t->token_stride < 0 || t->head_stride < 0) return "negative stride";
    // offsets in bytes stay within 63 bits
    const int64_t lim = INT64_MAX / 16;
    if (t->token_stride > lim / (tokens < 1 ? 1 : tokens) || t->head_stride > lim / t->heads) return "stride too large";
    if (tokens > 0 && (!t->data || ((uintptr_t)t->data & (uintptr_t)(dtype_bytes(t->dtype) - 1))))
        return "tensor data null or unaligned";
    if (out) {
        const int64_t n0 = t->heads, s0 = t->head_stride, n1 = tokens, s1 = t->token_stride;
        const bool apart = (n0 == 1 || s0 >= d) && (n1 <= 1 || s1 >= d) &&
                           (n0 == 1 || n1 <= 1 || s1 >= (n0 - 1) * s0 + d || s0 >= (n1 - 1) * s1 + d);
        if (!apart) return "an output's heads overlap";
    }
    return nullptr;
}

// heads of `t` start on 16-byte boundaries
inline bool wide_heads(const wici_heads *t) {
    const int per = 16 / dtype_bytes(t->dtype);
    return ((uintptr_t)t->data & 15) == 0 && t->token_stride % per == 0 && t->head_stride % per == 0;
}

// ---- shape of the row-wise kernels' launches ----
constexpr int kRowThreads = 128;
constexpr int kRowBlocks = 8;         // blocks on an SM: 64 registers a thread
constexpr int kBlockTokens = 8;       // tokens of a block at most

// Tokens of a block, a power of two: as many as leave two waves of blocks and more.
inline int tokens_of_block(int64_t tokens, int most, int sms) {
    int n = 1;
    while (2 * n <= most && tokens / (2 * n) >= 2 * kRowBlocks * sms) n *= 2;
    return n;
}

struct RowBlock {
    int tokens;                       // of a block: a power of two
    int rows;                         // of `chunks` lanes each, a multiple of `tokens`
};
// A block for rows of `chunks` lanes, `heads` of them a token: every token has a row of the block at least (rotated
// halves of 242 to 256 elements may take 17 lanes, which leaves 7 rows: 4 tokens), and no lanes are left without
// a row but those that fill the last warp (the shuffles of a row).
inline RowBlock row_block(int64_t tokens, int heads, int chunks, int sms) {
    const int most = kRowThreads / chunks;
    RowBlock b = {tokens_of_block(tokens, most < kBlockTokens ? most : kBlockTokens, sms), 0};
    const int need = (heads * b.tokens + 31) / 32 * 32;
    b.rows = most - most % b.tokens;
    b.rows = b.rows < need ? b.rows : need;
    return b;
}

inline bool words(const void *p) { return ((uintptr_t)p & 3) == 0; }   // of 32 bits; NULL among them

inline const char *check_rope(const wici_rope_plan *p) {
    if (!p) return "null rope plan";
    if (p->head_dim < 2 || p->head_dim > 256 || p->head_dim % 2 || p->rot_dim < 2 || p->rot_dim > p->head_dim ||
        p->rot_dim % 2 || (p->interleaved != 0 && p->interleaved != 1))
        return "rope plan was not made by wici_rope_make_plan";
    return nullptr;
}

}  // namespace wici
