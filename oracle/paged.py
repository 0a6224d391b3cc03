"""Oracle of the batched decode step's operators (test infrastructure only): rotary
positions with their scaling rules, the paged cache's 8- and 4-bit formats, and attention of one
token over a paged cache, each written from its definition in fp64.

A cache is held here as one entry per slot, not as bytes: `codes` [slots, 2, heads, d]
(values for bf16) and `scales` [slots, 2, heads] (None for bf16), slot = page * 16 + place;
`pack` lays it out as the library's pages.
"""
from __future__ import annotations

import numpy as np

PAGE = 16


# ------------------------------------------------------------------ rotary --
def rope_frequencies(rot, theta, scaling="none", factor=1.0, original_len=0, low=0.0, high=0.0):
    """Radians a position of each pair, and the gain."""
    f = np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":
        turns = original_len * f / (2 * np.pi)
        out = np.where(turns <= low, f / factor, f)
        mid = (turns > low) & (turns < high)
        t = (turns - low) / (high - low)
        return np.where(mid, f * ((1 - t) / factor + t), out), 1.0
    if scaling == "yarn":
        def pair_at(turns):
            return rot * np.log(original_len / (2 * np.pi * turns)) / (2 * np.log(theta))
        lo, hi = max(np.floor(pair_at(high)), 0), min(np.ceil(pair_at(low)), rot - 1)
        r = np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
        return f * (1 - r) + f / factor * r, 0.1 * np.log(factor) + 1.0
    return f, 1.0


def rope(x, positions, rot, freq, gain=1.0, interleaved=False, inverse=False):
    """x [tokens, heads, d] with its first `rot` elements of a head rotated, pair by pair."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    ang = np.asarray(positions, np.float64)[:, None] * freq[None]
    c, s = gain * np.cos(ang)[:, None], gain * np.sin(ang)[:, None]
    if inverse:
        s = -s
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        y[..., a] = x[..., a] * c[..., i] - x[..., b] * s[..., i]
        y[..., b] = x[..., a] * s[..., i] + x[..., b] * c[..., i]
    return y


# ----------------------------------------------------------- 8-bit formats --
def _e4m3_table():
    """The 256 values of e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities, S.1111.111 is NaN."""
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = np.nan if (b & 127) == 127 else (-v if b & 128 else v)
    return out


E4M3 = _e4m3_table()
_POSITIVE = E4M3[:127]


def e4m3_codes(v):
    """The nearest e4m3 value's byte, ties to the even mantissa; magnitudes above 448 give 448."""
    a = np.minimum(np.abs(np.asarray(v, np.float64)), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quantise(x, fmt):
    """(codes, scales) of heads x [..., d]; int8 codes as int8, e4m3 codes as bytes."""
    x = np.asarray(x, np.float64)
    top = 127.0 if fmt == "int8" else 448.0
    bad = ~np.isfinite(x).all(-1)
    scale = np.where(bad, 0, np.abs(np.where(np.isfinite(x), x, 0)).max(-1)) / top
    q = np.where(scale[..., None] > 0, np.where(bad[..., None], 0, x) / np.where(scale > 0, scale, 1)[..., None], 0)
    codes = np.rint(q).astype(np.int8) if fmt == "int8" else e4m3_codes(q)
    return codes, np.where(bad, np.nan, scale)


def code_values(codes, fmt):
    codes = np.asarray(codes)
    return codes.astype(np.float64) if fmt == "int8" else E4M3[codes.view(np.uint8)]


def block_bytes(fmt, d):
    return PAGE * d * 2 if fmt == "bf16" else PAGE * d + 4 * PAGE


def pack(codes, scales, fmt):
    """uint8 pages [pages][K|V][head] blocks from per-slot codes (bf16: uint16 bits) and scales."""
    slots, two, heads, d = codes.shape
    c = codes.reshape(slots // PAGE, PAGE, two, heads, d).transpose(0, 2, 3, 1, 4)
    c = np.ascontiguousarray(c)
    if fmt == "bf16":
        return c.view(np.uint8).reshape(-1)
    s = np.ascontiguousarray(scales.reshape(slots // PAGE, PAGE, two, heads).transpose(0, 2, 3, 1)).astype(np.float32)
    return np.concatenate([c.view(np.uint8).reshape(*c.shape[:3], -1), s.view(np.uint8).reshape(*c.shape[:3], -1)],
                          axis=-1).reshape(-1)


def unpack(data, heads, d, fmt):
    """The inverse of pack: (codes, scales)."""
    blocks = np.asarray(data).reshape(-1, 2, heads, block_bytes(fmt, d))
    pages = blocks.shape[0]

    def by_slot(a):
        return np.moveaxis(a, 3, 1).reshape(pages * PAGE, 2, heads, *a.shape[4:])

    if fmt == "bf16":
        c = np.ascontiguousarray(blocks).view(np.uint16).reshape(pages, 2, heads, PAGE, d)
        return by_slot(c), None
    c = blocks[..., :PAGE * d].reshape(pages, 2, heads, PAGE, d)
    s = np.ascontiguousarray(blocks[..., PAGE * d:]).view(np.float32)
    return by_slot(c.view(np.int8) if fmt == "int8" else c), by_slot(s)


# ------------------------------------------------------------ 4-bit format --
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])
E2M1_TOP, E2M1_LEAST = 2688.0, 2.0 ** -100          # 6 * 448; smaller scales are 0


def _nearest_code(a, unit, grid):
    """The place of the value of `grid` nearest to a / unit, the even one of two as near, by exact comparisons: a has 24
    significant bits, unit and grid's middles together at most 39."""
    middles = (grid[1:] + grid[:-1]) / 2
    code = np.zeros(np.broadcast(a, unit).shape, np.int64)
    for i, m in enumerate(middles):
        code += (a > m * unit) | ((a == m * unit) & (i % 2 == 1))
    return code


def quantise_e2m1(x):
    """(codes [..., d] in 0..15, e4m3 codes of blocks [..., d / 16], scales fp32) of heads x [..., d] that fp32 holds."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0, x)
    scale = (np.abs(x).max(-1) / E2M1_TOP).astype(np.float32)
    scale = np.where(scale < E2M1_LEAST, np.float32(0), scale)
    s = scale.astype(np.float64)[..., None]
    a = np.abs(x).reshape(*x.shape[:-1], -1, 16)
    each = np.where(s > 0, _nearest_code(a.max(-1), 6.0 * s, _POSITIVE), 0)
    unit = (E4M3[each] * s)[..., None]
    code = np.where(unit > 0, _nearest_code(a, unit, E2M1[:8]), 0)
    sign = np.where(np.signbit(x).reshape(a.shape) & (s > 0)[..., None], 8, 0)
    return (code | sign).reshape(x.shape).astype(np.uint8), each.astype(np.uint8), np.where(bad, np.float32(np.nan), scale)


def e2m1_values(codes, each, scales):
    v = E2M1[codes].reshape(*each.shape, 16) * E4M3[each][..., None]
    return v.reshape(codes.shape) * np.asarray(scales, np.float64)[..., None]


def pack_e2m1(codes, each, scales):
    """uint8 pages from per-slot codes [slots, 2, heads, d], block codes and scales."""
    def by_page(a):
        a = a.reshape(a.shape[0] // PAGE, PAGE, *a.shape[1:])
        return np.ascontiguousarray(np.moveaxis(a, 1, 3)).view(np.uint8).reshape(a.shape[0], 2, a.shape[3], -1)

    return np.concatenate([by_page(codes[..., 0::2] | codes[..., 1::2] << 4), by_page(each),
                           by_page(np.asarray(scales, np.float32))], axis=-1).reshape(-1)


def unpack_e2m1(data, heads, d):
    """The inverse of pack_e2m1."""
    row, each = d // 2, d // 16
    blocks = np.asarray(data).reshape(-1, 2, heads, PAGE * (row + each + 4))

    def by_slot(a, kind):
        a = np.ascontiguousarray(a).view(kind).reshape(*blocks.shape[:3], PAGE, -1)
        return np.moveaxis(a, 3, 1).reshape(blocks.shape[0] * PAGE, 2, heads, -1)

    c = by_slot(blocks[..., :PAGE * row], np.uint8)
    return (np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:3], d), by_slot(blocks[..., PAGE * row:PAGE * (row + each)], np.uint8),
            by_slot(blocks[..., PAGE * (row + each):], np.float32)[..., 0])


# --------------------------------------------------------------- attention --
def paged_attention(q, k, v, pages, lengths, scale, window=0):
    """q [batch, heads, d]; k, v [slots, kv heads, d]; one sequence, head and key after the other.
    Returns (out, lse, weight): weight[b, h] = sum_t p_t |v_t|, the size that rounding errors of p act on."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    B, H, d = q.shape
    group = H // k.shape[1]
    out, lse, weight = np.zeros((B, H, d)), np.full((B, H), -np.inf), np.zeros((B, H, d))
    for b in range(B):
        n = int(lengths[b])
        keys = range(max(0, n - window) if window else 0, n)
        slots = [int(pages[b][t // PAGE]) * PAGE + t % PAGE for t in keys]
        if not slots:
            continue
        for h in range(H):
            s = k[slots, h // group] @ q[b, h] * scale
            top = s.max()
            p = np.exp(s - top)
            lse[b, h] = top + np.log(p.sum())
            p = p / p.sum()
            out[b, h] = p @ v[slots, h // group]
            weight[b, h] = p @ np.abs(v[slots, h // group])
    return out, lse, weight


# -------------------------------------------------------- selection of pages --
def key_bounds(k):
    """(int8 codes [2, d], fp32 scale) of a page's keys [tokens, d], which fp32 holds: the largest and the smallest element
    by element over max |k| (1 / 127), whole numbers of fp32 quotients."""
    k = np.asarray(k, np.float32)
    if not np.isfinite(k).all():
        return np.zeros((2, k.shape[1]), np.int8), np.float32(np.nan)
    ends = np.stack((k.max(0), k.min(0)))
    scale = np.abs(ends).max() * (np.float32(1) / np.float32(127))
    if scale < np.float32(2.0 ** -126):
        return np.zeros_like(ends, np.int8), np.float32(0)
    return np.rint(ends / scale).astype(np.int8), scale


def page_scores(q, codes, scales):
    """fp32 scores [pages] of one KV head's query heads q [group, d] against codes [pages, 2, d] and scales [pages]."""
    q, best = np.asarray(q, np.float32), np.full(len(scales), -np.inf, np.float32)
    for x in q:
        m = np.abs(x).max()                                    # NaN where one is
        ok = np.isfinite(m) and m >= 2.0 ** -100
        w = [int(np.rint(v * (np.float32(1) / m * np.float32(1023)))) if ok else 0 for v in x]
        m = m if ok else np.float32(0)
        for p in range(len(scales)):
            dot = sum(w[d] * int(codes[p, 0 if w[d] > 0 else 1, d]) for d in range(len(w)))
            with np.errstate(over="ignore"):
                best[p] = max(best[p], np.float32(dot) * m)
    out = np.empty(len(scales), np.float32)
    for p, s in enumerate(scales):
        with np.errstate(over="ignore"):
            out[p] = np.inf if not np.isfinite(s) else np.float32(0) if s == 0 else best[p] * s
    return out


def selected_pages(scores, keep, first, recent):
    """The columns of the selected pages, ascending."""
    n = len(scores)
    if n <= keep:
        return list(range(n))
    forced = [p for p in range(n) if p < first or p >= n - recent]
    rest = sorted((p for p in range(n) if p not in set(forced)), key=lambda p: (-float(scores[p]), p))
    return sorted(forced + rest[:keep - len(forced)])
