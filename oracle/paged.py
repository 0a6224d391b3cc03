"""Oracle of the batched decode step's operators (test infrastructure only): rotary
positions with their scaling rules, the paged cache's 8-bit formats, and attention of one
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
