/*
 * wici_ops.h - operators of a batched decode step, for engines that own their
 * device memory: rotary positions, writing and reading a paged key-value cache
 * (bf16, or quantised to 8 bits), and attention of one new token per sequence
 * over that cache.  They stand beside wici_lm_head_argmax_noalloc (wici.h) and
 * need no context; wici_kv_view hands them the cache of one.
 *
 * A step of one layer for a batch of clients: the q|k|v projection, then
 * wici_kv_append (rotates q and k, writes k and v), then wici_paged_attention.
 *
 * Conventions for every entry point
 *   - Return value as in wici.h; messages are in wici_last_error(NULL).  On
 *     WICI_E_ARG nothing has been launched.
 *   - Work is enqueued on cuda_stream (a cudaStream_t, NULL for the legacy
 *     stream) of the current device and the call does not synchronise; every
 *     device pointer belongs to that device.  Every launch can be captured into
 *     a CUDA graph (make a device's first wici_paged_attention or
 *     wici_paged_attention_workspace_bytes before the capture).  No call allocates.
 *   - What the host cannot check without a copy (slots, page numbers, lengths)
 *     is checked by the kernels: nothing outside the cache is read or written,
 *     and `status` (device int32, may be NULL) collects WICI_BAD_* bits.  The
 *     library only sets bits; the caller clears the word before first use.
 *   - Tensors overlap only where a call says so.
 */
#ifndef WICI_OPS_H
#define WICI_OPS_H

#include "wici.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of activations. */
typedef enum wici_dtype { WICI_BF16 = 0, WICI_F16 = 1, WICI_F32 = 2 } wici_dtype;

/* Bits of a status word. */
enum {
    WICI_BAD_SLOT = 1,    /* a slot >= 16 * n_pages: the token was not written, or read as NaN */
    WICI_BAD_PAGE = 2,    /* a needed page number outside [0, n_pages): the sequence's output is NaN */
    WICI_BAD_LENGTH = 4   /* a length > 16 * max_pages: the sequence's output is NaN */
};

/* A caller's tensor [tokens][heads][head_dim], elements of a head adjacent.
 * Strides are in elements, not negative, and for an output no two elements may
 * share a place.  Any alignment that is the type's own; 16-byte aligned heads
 * take the wide path. */
typedef struct wici_heads {
    void *data;
    int64_t token_stride, head_stride;
    int32_t heads;
    int32_t dtype;        /* wici_dtype */
} wici_heads;

/* ------------------------------------------------------------ rotary positions
 * Pair i < rot_dim / 2 of a head at position p turns by the angle p f_i,
 *   y_a = g (x_a cos - x_b sin),  y_b = g (x_a sin + x_b cos),
 * with (a, b) = (i, i + rot_dim / 2), or (2i, 2i + 1) when interleaved; elements
 * from rot_dim on are copied.  f_i = theta^(-2i / rot_dim), then by `scaling`:
 *   WICI_ROPE_LINEAR  f / factor
 *   WICI_ROPE_BANDS   t = original_len f / 2 pi (turns in the original context):
 *                     f / factor where t <= low, f where t >= high, linear in t
 *                     between (the Llama-3 rule: low 1, high 4, factor 8)
 *   WICI_ROPE_YARN    with c(b) = rot_dim ln(original_len / 2 pi b) / (2 ln theta),
 *                     lo = max(floor c(high), 0), hi = min(ceil c(low), rot_dim - 1),
 *                     r = clamp((i - lo) / max(hi - lo, 0.001), 0, 1):
 *                     f (1 - r) + f r / factor   (Peng et al. 2023: low 1, high 32)
 * g is `gain`, or where that is 0: 1, and 0.1 ln(factor) + 1 for YaRN.  The
 * paper has no counterpart; the contexts of wici.h run the unscaled half layout. */
enum { WICI_ROPE_NONE = 0, WICI_ROPE_LINEAR = 1, WICI_ROPE_BANDS = 2, WICI_ROPE_YARN = 3 };

typedef struct wici_rope_spec {
    double theta;             /* > 1 */
    double factor;            /* >= 1; 1 without scaling */
    double low, high;         /* BANDS, YARN: 0 < low < high */
    double gain;              /* >= 0 */
    int32_t original_len;     /* BANDS, YARN: >= 1 */
    int32_t head_dim;         /* 2..256, even */
    int32_t rot_dim;          /* 2..head_dim, even */
    int32_t interleaved;      /* 0 or 1 */
    int32_t scaling;          /* WICI_ROPE_* */
} wici_rope_spec;

/* Filled once by wici_rope_make_plan (a host call), then read by any number of
 * calls on any device.  turns[i] is f_i / 2 pi as a 64-bit fraction of a turn:
 * position times turns[i] modulo 2^64 is the angle, exact at any int32 position. */
typedef struct wici_rope_plan {
    uint64_t turns[128];
    float gain;
    int32_t head_dim, rot_dim, interleaved;
} wici_rope_plan;

int wici_rope_make_plan(const wici_rope_spec *spec, wici_rope_plan *plan);

/* y = x rotated by `positions` (device int32[tokens], any value), computed in
 * fp32 and rounded once.  inverse = 1 turns by -p f_i with the same g: the
 * gradient with respect to x of a rotation whose gradient is given.  x and y
 * have one type and the same heads; y may be x itself (same data and strides). */
int wici_rope(void *cuda_stream, const wici_rope_plan *plan, int32_t inverse, const int32_t *positions,
              int64_t tokens, const wici_heads *x, const wici_heads *y);

/* --------------------------------------------------------- paged key-value cache
 * n_pages pages of 16 tokens, page_stride bytes apart, each [K|V][kv head] blocks:
 *   WICI_KV_BF16  bf16 [16][head_dim]           (a context's own layout, wici_get_sizes)
 *   WICI_KV_INT8  int8 [16][head_dim], then fp32 scale[16]
 *   WICI_KV_E4M3  e4m3 [16][head_dim], then fp32 scale[16]
 * A token's head stands for code * scale; it is written with scale = max|x| / 127
 * (int8) or / 448 (e4m3) in fp32 and code = x / scale rounded to nearest even (for
 * e4m3 from the fp32 quotient, which is right to its last bit).  A
 * head whose scale would be below 2^-126, one of zeros among them, has scale 0, and
 * one that holds an infinity or NaN has scale NaN (it reads as NaN throughout).
 * Slot s is place s % 16 of page s / 16.  The paper names no cache precision; 8-bit
 * codes halve the bytes that bound decoding. */
enum { WICI_KV_BF16 = 0, WICI_KV_INT8 = 1, WICI_KV_E4M3 = 2 };

typedef struct wici_kv_cache {
    void *data;               /* 16-byte aligned */
    int64_t page_stride;      /* bytes, a multiple of 16, at least wici_kv_page_bytes */
    int32_t n_pages;          /* 1 .. 2^27 - 1 */
    int32_t n_kv_heads;       /* 1 .. 1024 */
    int32_t head_dim;         /* 64 or 128 */
    int32_t format;           /* WICI_KV_* */
} wici_kv_cache;

/* Bytes of one page (0 for an unknown format or a head_dim that is not 64 or 128). */
int64_t wici_kv_page_bytes(int32_t format, int32_t n_kv_heads, int32_t head_dim);

/* Write k and v (n_kv_heads heads, one type) of `tokens` tokens at `slots`
 * (device int32[tokens]; a negative one is skipped: the padding of a fixed-size
 * batch).  Slots >= 0 are distinct within a call.  With `rope` (head_dim the
 * cache's, rot_dim a multiple of 16), k is rotated by `positions` on the way, and
 * so is q into q_out (both or neither; any number of heads; k's type; q_out may
 * be q itself), skipped tokens included.  Without `rope`, positions, q and q_out
 * are NULL. */
int wici_kv_append(void *cuda_stream, const wici_kv_cache *cache, const int32_t *slots, int64_t tokens,
                   const wici_heads *k, const wici_heads *v, const wici_rope_plan *rope, const int32_t *positions,
                   const wici_heads *q, const wici_heads *q_out, int32_t *status);

/* k[i], v[i] (outputs; either may be NULL) = the values at slots[i], code * scale in
 * fp32 and that rounded to the output's type; zeros where slots[i] < 0.  Slots may
 * repeat. */
int wici_kv_read(void *cuda_stream, const wici_kv_cache *cache, const int32_t *slots, int64_t tokens,
                 const wici_heads *k, const wici_heads *v, int32_t *status);

/* Attention of one new token per sequence: for sequence b and query head h,
 * which reads KV head h / (heads / n_kv_heads),
 *   s_t = scale q.k_t,  out = sum_t e^(s_t - lse) v_t,  lse = ln sum_t e^(s_t)
 * over its keys t in [max(0, n - window), n) (window 0: all), n = lengths[b]; key t
 * is place t % 16 of page pages[b * max_pages + t / 16].  Pages of other keys are
 * not read and may hold anything.  A sequence without keys (n <= 0) has out 0 and
 * lse -infinity.  Infinities and NaNs in a sequence's own keys act as in the
 * formula, in its own result alone (e^(s_t - max s) below 2^-126 counts as 0).
 * Over an 8-bit cache a key's weight times its scale of V is held to 2^-22 of itself
 * or 2^-32 of the sequence's largest, far less than what codes cost that key's values.
 * Several sequences may share pages. */
typedef struct wici_attn_shape {
    int32_t batch;            /* 0 .. 65535 */
    int32_t max_pages;        /* columns of `pages`, 1 .. 2^27 - 1; (max_pages + 2) * heads < 2^31 */
    int32_t window;           /* >= 0 */
    float scale;              /* finite */
} wici_attn_shape;

enum { WICI_ATTN_ZEROED = 16384 };

/* Bytes of the workspace on the current device for up to `batch` sequences and
 * n_q_heads query heads. */
int wici_paged_attention_workspace_bytes(const wici_kv_cache *cache, int32_t n_q_heads, int32_t batch, size_t *bytes);

/* q and out: `batch` tokens of n_q_heads heads (a multiple of n_kv_heads), each of
 * its own type; out rows past the batch are left as they are.  lse: device
 * fp32 [batch][n_q_heads], or NULL.  workspace: 16-byte aligned, its first
 * WICI_ATTN_ZEROED bytes zeroed once by the caller before its first use; calls that share one must be ordered on one stream
 * (a captured graph needs one of its own unless its launches are ordered with every
 * other user's). */
int wici_paged_attention(void *cuda_stream, const wici_kv_cache *cache, const wici_attn_shape *shape,
                         const int32_t *pages, const int32_t *lengths, const wici_heads *q, const wici_heads *out,
                         float *lse, void *workspace, int32_t *status);

/* The cache of layer `layer` of a context, as of the work already enqueued on the
 * context's stream, and its page table (device int32[pages], logical -> physical;
 * *n_logical entries).  Both stay valid until wici_destroy; the first wici_kv_len
 * positions hold tokens.  Read it on the context's stream or after it; what the
 * context wrote is the context's, and is not to be written. */
int wici_kv_view(const wici_ctx *ctx, int32_t layer, wici_kv_cache *cache, const int32_t **pages, int32_t *n_logical);

#ifdef __cplusplus
}
#endif

#endif /* WICI_OPS_H */
