"""The operators of a batched decode step (include/wici_ops.h) through their binding against
the fp64 oracle (oracle/paged.py).

Tolerances, from the arithmetic:
* storing to a type: half a step, eps / 2 of the value (plus half the smallest fp16 step).
* a rotation in fp32: the angle's rest of at most pi / 4 is off by 2^-24 of itself (a conversion) and 2^-30 turns,
  sincospif by two units in the last place, the gain's product and each product and sum by half one: below
  2^-21 (|x_a| + |x_b|) g.
* a code: x / scale has to round as in 64 bits unless it lies within `near` of a border: 127 * 2^-22 for given
  values (quotient and scale rounded to fp32), and for rotated ones, off by 2^-21 (|x_a| + |x_b|) <= 2^-20 * 1.42 amax
  in x as well as in the scale: 127 * 2^-18.  e4m3 borders are relative: the same with 1 in place of 127.
* attention: a product q.k is off by 2 d 2^-23 of the sum of its |products| (tensor cores may truncate each
  add) and by 2^-16 of it where q has more bits than two 16-bit terms hold; probabilities carry at least 16 bits and
  the exponential is good to 2^-21; sums over n keys add n 2^-23.  All act on sum p |v|.
"""
import numpy as np
import pytest

from oracle import paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import gen  # noqa: E402
import oracle  # noqa: E402
from paper_2608_24204_gb300 import PagedKV, Rope, WiciModel, ops, wici  # noqa: E402

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(a):
    return torch.tensor(np.asarray(a, np.int32), device="cuda")


def half_step(v, dtype):
    return np.abs(v) * (torch.finfo(DT[dtype]).eps / 2) * (1 + 2.0 ** -10) + (2.0 ** -25 if dtype == "f16" else 0)


def within(got, want, tol, what):
    got, want = np.asarray(got), np.asarray(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaNs"
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want) | np.isnan(want))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax((np.abs(got - want) / tol)[bad]):.2f} x the tolerance"


def randn(rng, *shape, dtype="f32", scale=1.0):
    return torch.tensor(rng.normal(size=shape) * scale, device="cuda").to(DT[dtype])


SCALED = {"none": {}, "linear": {"factor": 4.0}, "bands": {"factor": 8.0, "original_len": 512, "low": 1.0, "high": 4.0},
          "yarn": {"factor": 16.0, "original_len": 512, "low": 1.0, "high": 32.0}}


# ------------------------------------------------------------------- rotary --
def check_rope(x, y, pos, rot, theta, interleaved, scaling, inverse, dtype):
    f, g = paged.rope_frequencies(rot, theta, scaling, **SCALED[scaling])
    want = paged.rope(f64(x), pos, rot, f, g, interleaved, inverse)
    ax = np.abs(f64(x))
    mix = np.zeros_like(ax)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    mix[..., a] = mix[..., b] = ax[..., a] + ax[..., b]
    within(f64(y), want, 2.0 ** -21 * g * mix + half_step(want, dtype), "rope")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,heads,d,rot,interleaved,scaling,inverse", [
    (1, 1, 128, 128, False, "none", False),
    (1, 40, 128, 128, False, "bands", False),
    (7, 3, 64, 64, True, "linear", False),
    (33, 5, 128, 64, False, "yarn", True),
    (19, 2, 80, 20, True, "yarn", False),       # odd sizes: element-wise accesses
    (5, 9, 2, 2, False, "none", False),
    (4, 3, 256, 250, False, "bands", True),
    (300, 33, 96, 96, False, "none", False),
    (2000, 8, 32, 16, True, "none", True),
])
def test_rope(dtype, tokens, heads, d, rot, interleaved, scaling, inverse):
    rng = np.random.default_rng(tokens * 1000 + d)
    pos = rng.integers(-3, 1 << 20, tokens)
    x = randn(rng, tokens, heads, d, dtype=dtype)
    kept = x.clone()
    r = Rope(d, 5e5, rot_dim=rot, interleaved=interleaved, scaling=scaling, **SCALED[scaling])
    y = r.apply(x, ints(pos), inverse=inverse)
    assert torch.equal(x, kept)
    check_rope(x, y, pos, rot, 5e5, interleaved, scaling, inverse, dtype)
    z = r.apply(x, ints(pos), out=x, inverse=inverse)        # in place
    assert z is x and torch.equal(x, y)


@pytest.mark.parametrize("layout", ["packed", "heads first", "unaligned", "broadcast tokens"])
def test_rope_strides(layout):
    rng = np.random.default_rng(3)
    T, H, d = 37, 4, 64
    if layout == "packed":
        x = randn(rng, T, H + 3, d, dtype="bf16")[:, 1:1 + H]
        y = torch.full((T, H + 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
        out = y[:, 2:]
    elif layout == "heads first":
        x = randn(rng, H, T, d, dtype="bf16").transpose(0, 1)
        y = torch.full((H, T + 5, d), 7.0, dtype=torch.bfloat16, device="cuda")
        out = y[:, :T].transpose(0, 1)
    elif layout == "unaligned":
        x = randn(rng, T * H * d + 1, dtype="bf16")[1:].view(T, H, d)
        y = torch.full((T * H * d + 3,), 7.0, dtype=torch.bfloat16, device="cuda")
        out = y[3:].view(T, H, d)
    else:
        x = randn(rng, 1, H, d, dtype="bf16").expand(T, H, d)
        y = out = torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    pos = rng.integers(0, 5000, T)
    Rope(d, 1e4).apply(x, ints(pos), out=out)
    check_rope(x, out, pos, d, 1e4, False, "none", False, "bf16")
    assert int((y == 7.0).sum()) >= y.numel() - out.numel()  # nothing beside the output was written
    out.fill_(7.0)
    assert bool((y == 7.0).all())


def test_rope_of_extreme_positions_and_values():
    rng = np.random.default_rng(4)
    pos = np.array([-2 ** 31, 2 ** 31 - 1, 2 ** 24 + 1, 123456789, 0, -1])
    x = randn(rng, 6, 2, 128)
    check_rope(x, Rope(128, 5e5).apply(x, ints(pos)), pos, 128, 5e5, False, "none", False, "f32")
    x[1, 0, 3], x[2, 1, 70] = float("inf"), float("nan")
    y = Rope(128, 5e5).apply(x, ints(pos))
    touched = torch.zeros(6, 2, 128, dtype=torch.bool, device="cuda")
    touched[1, 0, [3, 67]] = touched[2, 1, [70, 6]] = True
    assert bool(torch.isfinite(y[~touched]).all()) and not bool(torch.isfinite(y[touched]).any())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,d,rot", [
    (1, 1, 8, 2), (1, 40, 128, 126), (5, 33, 80, 20), (7, 2, 96, 6), (3, 70, 4, 4), (9, 3, 132, 70), (6, 2, 256, 254),
    (2, 5, 72, 50), (11, 4, 64, 40), (5000, 3, 16, 10), (3001, 7, 40, 36),
])
def test_rope_of_ragged_rotations(dtype, interleaved, tokens, heads, d, rot):
    # rotated parts that end, or meet, anywhere in a 16-byte word; an output row with gaps that have to stay
    rng = np.random.default_rng(tokens + d + rot)
    pos = rng.integers(-3, 1 << 20, tokens)
    x = randn(rng, tokens, heads, d, dtype=dtype)
    # infinities and NaNs touch their own pair alone, and behind the rotated part themselves
    wild = torch.zeros(tokens, heads, d, dtype=torch.bool, device="cuda")
    places = ({0, 1} if interleaved else {0, rot // 2}) | ({rot} if rot < d else set())
    wild[tokens // 2, heads - 1, sorted(places)] = True
    x[tokens // 2, heads - 1, 0] = float("inf")
    if rot < d:
        x[tokens // 2, heads - 1, rot] = float("nan")
    y = torch.full((tokens, heads + 1, d + 8), 7.0, dtype=DT[dtype], device="cuda")
    r = Rope(d, 5e5, rot_dim=rot, interleaved=interleaved)
    out = y[:, :heads, :d]
    r.apply(x, ints(pos), out=out)
    assert bool((y[:, heads] == 7.0).all()) and bool((y[..., d:] == 7.0).all())
    assert not bool(torch.isfinite(out[wild]).any()) and bool(torch.isfinite(out[~wild]).all())
    tame = x.masked_fill(wild, 1.0)
    check_rope(tame, r.apply(tame, ints(pos)), pos, rot, 5e5, interleaved, "none", False, dtype)
    assert torch.equal(r.apply(tame, ints(pos))[~wild], out[~wild])
    want = r.apply(tame, ints(pos), inverse=True)
    assert torch.equal(r.apply(tame, ints(pos), out=tame, inverse=True), want)      # in place
    check_rope(x.masked_fill(wild, 1.0), want, pos, rot, 5e5, interleaved, "none", True, dtype)


def test_rope_inverse_is_the_gradient_by_differences():
    # L = sum(w * rope(x)): dL/dx by central differences in x of the fp64 oracle, at step 1 (the map is linear)
    rng = np.random.default_rng(5)
    T, d, rot = 3, 32, 24
    r = Rope(d, 1e4, rot_dim=rot, interleaved=True, scaling="yarn", **SCALED["yarn"])
    f, g = paged.rope_frequencies(rot, 1e4, "yarn", **SCALED["yarn"])
    pos = np.array([2, 900, 77])
    x, w = rng.normal(size=(T, 1, d)), rng.normal(size=(T, 1, d))
    got = f64(r.apply(torch.tensor(w, device="cuda").float(), ints(pos), inverse=True))
    for i in range(d):
        e = np.zeros((1, 1, d))
        e[..., i] = 1.0
        up, down = (paged.rope(x + s * e, pos, rot, f, g, True) for s in (0.5, -0.5))
        want = (w * (up - down)).sum((1, 2))
        assert np.all(np.abs(got[:, 0, i] - want) <= 2.0 ** -20 * g * np.abs(w).max())


# ------------------------------------------------------------- append, read --
def near_border(x, scale, fmt, near):
    """Where x / scale lies within `near` of a value that rounds either way."""
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.nan_to_num(np.abs(x) / scale[..., None])
    if fmt == "int8":
        return np.abs(q - np.floor(q) - 0.5) <= 127 * near
    grid = paged.E4M3[:127]
    mid = (grid[1:] + grid[:-1]) / 2
    j = np.clip(np.searchsorted(mid, q), 1, 125)
    return np.minimum(np.abs(q - mid[j]), np.abs(q - mid[j - 1])) <= near * np.maximum(q, 2.0 ** -9) * 2


def check_written(data, slots, k, v, fmt, d, kv, before, rotated, g=1.0):
    """The cache bytes after an append of k, v (fp64 [tokens, kv, d], rotated in 64 bits) at slots."""
    codes, scales = paged.unpack(data.cpu().numpy(), kv, d, fmt)
    old_codes, old_scales = paged.unpack(before.cpu().numpy(), kv, d, fmt)
    live = slots >= 0
    others = np.ones(codes.shape[0], bool)
    others[slots[live]] = False
    np.testing.assert_array_equal(codes[others], old_codes[others])
    if scales is not None:
        np.testing.assert_array_equal(scales[others].view(np.uint32), old_scales[others].view(np.uint32))
    for which, x in ((0, k), (1, v)):
        x, got = x[live], codes[slots[live], which]
        turned = rotated and which == 0
        slack = 2.0 ** -20 * 1.42 * g * np.abs(x).max(-1, keepdims=True) if turned else 0
        if fmt == "bf16":
            val = (got.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
            within(val, x, half_step(x, "bf16") + slack, "bf16 cache")
            continue
        s = scales[slots[live], which]
        want_codes, want_s = paged.quantise(x, fmt)
        within(s, want_s, want_s * (2.0 ** -18 if turned else 2.0 ** -23), "scale")
        gv, wv = paged.code_values(got, fmt), paged.code_values(want_codes, fmt)
        near = near_border(x, want_s, fmt, 2.0 ** -18 if turned else 2.0 ** -22)
        same = gv == wv
        assert np.all(same | near), f"{fmt}: {(~(same | near)).sum()} codes differ away from a border"
        step = 1.0 if fmt == "int8" else 2.0 ** -3 * np.maximum(np.abs(wv), 2.0 ** -6) * 2
        assert np.all(np.abs(gv - wv) <= step)


def slots_for(rng, tokens, pages):
    s = rng.permutation(pages * 16)[:tokens]
    return s.astype(np.int64)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype,tokens,kv,d,q_heads,rot,scaling,interleaved", [
    ("bf16", 1, 8, 128, 32, 128, "bands", False),
    ("f32", 1, 1, 64, 0, 0, "none", False),
    ("f16", 17, 2, 64, 6, 64, "none", True),
    ("bf16", 100, 3, 128, 15, 64, "yarn", False),
    ("f32", 333, 8, 128, 8, 128, "linear", False),
    ("f16", 50, 5, 128, 0, 0, "none", False),
    ("bf16", 1000, 4, 64, 0, 32, "none", True),      # k rotated without a q
])
def test_append_and_read(fmt, dtype, tokens, kv, d, q_heads, rot, scaling, interleaved):
    rng = np.random.default_rng(tokens + d)
    pages = tokens // 16 + 3
    before = torch.tensor(rng.integers(0, 256, pages * ops.wici_kv_page_bytes(ops.FORMATS[fmt], kv, d)), dtype=torch.uint8,
                          device="cuda")
    cache = PagedKV(kv, d, fmt, data=before.clone())
    k, v = randn(rng, tokens, kv, d, dtype=dtype, scale=3.0), randn(rng, tokens, kv, d, dtype=dtype)
    if tokens > 3:
        v[1] = 0                                              # a head of zeros
        k[2, 0] *= 2.0 ** -10
    slots = slots_for(rng, tokens, pages)
    if tokens > 5:
        slots[[3, tokens - 1]] = [-1, -7]                      # padding
    pos = rng.integers(0, 100000, tokens)
    kw, g, k64 = {}, 1.0, f64(k)
    if rot:
        r = Rope(d, 5e5, rot_dim=rot, interleaved=interleaved, scaling=scaling, **SCALED[scaling])
        f, g = paged.rope_frequencies(rot, 5e5, scaling, **SCALED[scaling])
        kw = {"rope": r, "positions": ints(pos)}
        k64 = paged.rope(k64, pos, rot, f, g, interleaved)
        if q_heads:
            kw["q"] = randn(rng, tokens, q_heads, d, dtype=dtype)
    q_out = cache.append(k, v, ints(slots), **kw)
    cache.check()
    check_written(cache.data, slots, k64, f64(v), fmt, d, kv, before, bool(rot), g)
    if q_heads:
        check_rope(kw["q"], q_out, pos, rot, 5e5, interleaved, scaling, False, dtype)
    codes, scales = paged.unpack(cache.data.cpu().numpy(), kv, d, fmt)
    back = np.concatenate([slots[::-1], slots[:2], [-3]])     # any order, repeats, padding
    for out_dtype in DT:
        got = cache.read(ints(back), dtype=DT[out_dtype])
        for which in (0, 1):
            c = codes[back, which]
            if fmt == "bf16":
                want = (c.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
            else:
                want = paged.code_values(c, fmt) * scales[back, which][..., None].astype(np.float64)
            want[back < 0] = 0
            if out_dtype == "f16":
                want = np.where(np.abs(want) >= 65520, np.sign(want) * np.inf, want)
            within(f64(got[which]), want, half_step(want, out_dtype) + 2.0 ** -24 * np.abs(want), f"read {out_dtype}")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_of_infinities_nans_and_tiny_heads(fmt):
    k = torch.ones(5, 1, 64, device="cuda")
    k[0, 0, 5], k[1, 0, 63], k[2] = float("inf"), float("nan"), 1e-40
    k[3] = 1e-30
    cache = PagedKV(1, 64, fmt, n_pages=1)
    cache.append(k, -k, ints(range(5)))
    kk, vv = (f64(t)[:, 0] for t in cache.read(ints(range(5)), dtype=torch.float32))
    assert np.isnan(kk[:2]).all() and np.isnan(vv[:2]).all()
    assert np.all((kk[2] >= 0) & (kk[2] <= 2e-40))            # below the normal range: codes are coarse, not wild
    np.testing.assert_allclose(kk[3], 1e-30, rtol=2.0 ** -21)  # the largest magnitude takes the largest code
    np.testing.assert_allclose(kk[4], 1.0, rtol=2.0 ** -22)
    np.testing.assert_array_equal(vv[2:], -kk[2:])


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_bad_slots_write_nothing_read_nan_and_are_reported(fmt):
    cache = PagedKV(2, 64, fmt, n_pages=2)
    k = torch.ones(4, 2, 64, device="cuda")
    slots = ints([0, 32, 2 ** 31 - 1, 31])
    cache.append(k, k, slots)
    with pytest.raises(wici.WiciError, match="slot"):
        cache.check()
    cache.check()                                             # cleared
    codes, _ = paged.unpack(cache.data.cpu().numpy(), 2, 64, fmt)
    assert [int(s) for s in np.nonzero(codes.reshape(32, -1).any(-1))[0]] == [0, 31]
    got, _ = cache.read(slots, dtype=torch.float32)
    with pytest.raises(wici.WiciError, match="slot"):
        cache.check()
    assert bool(torch.isnan(got[1:3]).all()) and bool(((got[[0, 3]] - 1).abs() < 2.0 ** -20).all())


def test_read_of_one_side_into_strided_outputs():
    rng = np.random.default_rng(6)
    cache = PagedKV(3, 64, "e4m3", n_pages=4)
    x = randn(rng, 60, 3, 64)
    cache.append(x, 2 * x, ints(range(60)))
    both = cache.read(ints(range(60)), dtype=torch.float32)
    wide = torch.full((3, 61, 65), 7.0, device="cuda")
    out = wide[:, :60, :64].transpose(0, 1)                   # heads first, unaligned rows
    st = torch.cuda.current_stream().cuda_stream
    slots = ints(range(60))
    for which in (0, 1):
        hs = ops.heads_of(out, 64, out.device, "out")
        ops.wici_kv_read(st, cache.cache, slots.data_ptr(), 60, *((hs, None) if which == 0 else (None, hs)))
        assert torch.equal(out, both[which])
    assert bool((wide[:, 60] == 7.0).all()) and bool((wide[:, :, 64] == 7.0).all())


# ---------------------------------------------------------------- attention --
def attention_case(rng, B, kv, group, d, fmt, dtype, lengths, max_pages=None, spread=1.0, poison=True):
    """A cache whose used slots hold values and whose every other byte is set (NaN in each format), q, pages."""
    lengths = np.asarray(lengths)
    need = [(max(int(n), 0) + 15) // 16 for n in lengths]
    total = sum(need) + 2
    slots = total * 16
    values = rng.normal(size=(slots, 2, kv, d)) * np.exp(0.5 * rng.normal(size=(2, kv, d)))
    values[:, 1] += 0.2
    if fmt == "bf16":
        codes = f64(torch.tensor(values).to(torch.bfloat16))
        codes = torch.tensor(codes).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
        scales, vals = None, (codes.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    else:
        codes, scales = paged.quantise(values, fmt)
        scales = scales.astype(np.float32)
        vals = paged.code_values(codes, fmt) * scales[..., None].astype(np.float64)
    order = rng.permutation(total)
    pages = np.full((len(lengths), max_pages or max(max(need), 1)), -1)
    used = np.zeros(slots, bool)
    at = 0
    for b, n in enumerate(need):
        pages[b, :n] = order[at:at + n]
        for t in range(max(int(lengths[b]), 0)):
            used[pages[b, t // 16] * 16 + t % 16] = True
        at += n
    if poison:
        codes = codes.copy()
        codes[~used] = np.array(0xFFFF if fmt == "bf16" else 0xFF, np.uint16 if fmt == "bf16" else np.uint8).astype(codes.dtype)
        if scales is not None:
            scales[~used] = np.nan
    data = torch.tensor(paged.pack(codes, scales, fmt), device="cuda")
    q = randn(rng, len(lengths), kv * group, d, dtype=dtype, scale=spread)
    return PagedKV(kv, d, fmt, data=data), q, pages, vals


def check_attention(cache, q, pages, lengths, vals, scale, window, out, lse, dtype, out_dtype=None):
    d = q.shape[-1]
    q64 = f64(q)
    want, want_lse, weight = paged.paged_attention(q64, vals[:, 0], vals[:, 1], pages, lengths, scale, window)
    for b in range(q.shape[0]):
        n = max(int(lengths[b]), 0)
        if n == 0:
            assert bool((out[b] == 0).all()) and (lse is None or bool((lse[b] == -np.inf).all()))
            continue
        keys = range(max(0, n - window) if window else 0, n)
        slots = [int(pages[b][t // 16]) * 16 + t % 16 for t in keys]
        for h in range(q.shape[1]):
            kk = vals[slots, 0, h // (q.shape[1] // vals.shape[2])]
            size = float(np.max(np.abs(kk) @ np.abs(q64[b, h])) * abs(scale))
            ds = size * (2 * d * 2.0 ** -23 + (2.0 ** -16 if dtype == "f32" else 0.0))
            rel = 2 * ds + 2.0 ** -16 + 2.0 ** -21 + len(slots) * 2.0 ** -23
            within(f64(out[b, h]), want[b, h], rel * weight[b, h] + half_step(want[b, h], out_dtype or dtype) + 1e-30,
                   f"attention of sequence {b}, head {h}")
            if lse is not None:
                within(float(lse[b, h]), want_lse[b, h], ds + 2.0 ** -20 + len(slots) * 2.0 ** -23 + 2.0 ** -23 * abs(want_lse[b, h]),
                       f"lse of sequence {b}, head {h}")


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("dtype,kv,group,d,lengths,window", [
    ("bf16", 1, 1, 128, [1], 0),
    ("f32", 2, 4, 64, [0, 1, 2, 15, 16, 17, 31, 33], 0),
    ("bf16", 8, 4, 128, [300, 0, 129, 1, 128, 127], 0),
    ("f16", 3, 5, 128, [70, 257, 16], 0),
    ("f32", 1, 8, 128, [1000, 3], 0),
    ("bf16", 2, 16, 64, [200, 90], 0),
    ("bf16", 1, 71, 64, [40, 150, 0], 0),
    ("f32", 2, 7, 128, [500, 64, 20, 0, 1], 33),
    ("bf16", 4, 2, 64, [400, 399, 385, 384], 16),
    ("f16", 1, 9, 128, [333, 18], 1),
])
def test_attention(fmt, dtype, kv, group, d, lengths, window):
    rng = np.random.default_rng(len(lengths) * 100 + group)
    cache, q, pages, vals = attention_case(rng, len(lengths), kv, group, d, fmt, dtype, lengths)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    for out_dtype in {dtype, "f32"}:
        out = torch.full(q.shape, 7.0, dtype=DT[out_dtype], device="cuda")
        cache.attend(q, ints(pages), ints(lengths), window=window, out=out, lse=lse)
        cache.check()
        check_attention(cache, q, pages, lengths, vals, d ** -0.5, window, out, lse, dtype, out_dtype)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_attention_over_a_long_cache_of_few_sequences(fmt):
    # one KV head: the length is what the work is split over
    rng = np.random.default_rng(11)
    lengths = [9001, 5]
    cache, q, pages, vals = attention_case(rng, 2, 1, 2, 128, fmt, "bf16", lengths, max_pages=700)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = cache.attend(q, ints(pages), ints(lengths), lse=lse)
    check_attention(cache, q, pages, lengths, vals, 128 ** -0.5, 0, out, lse, "bf16")
    for window in (8999, 4000, 100):
        out = cache.attend(q, ints(pages), ints(lengths), window=window, lse=lse)
        check_attention(cache, q, pages, lengths, vals, 128 ** -0.5, window, out, lse, "bf16")


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_attention_of_many_ragged_sequences(fmt):
    rng = np.random.default_rng(12)
    lengths = rng.integers(0, 120, 300)
    lengths[[5, 299]] = 0
    cache, q, pages, vals = attention_case(rng, 300, 1, 2, 64, fmt, "bf16", lengths)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = cache.attend(q, ints(pages), ints(lengths), lse=lse)
    check_attention(cache, q, pages, lengths, vals, 0.125, 0, out, lse, "bf16")


@pytest.mark.parametrize("fmt,d,unit", [("bf16", 128, 16), ("int8", 64, 64), ("e4m3", 128, 32)])
@pytest.mark.parametrize("kv,group,tail", [(1, 1, 0), (3, 2, 900), (4, 16, 0)])
def test_attention_of_short_sequences_beside_long_ones(fmt, d, unit, kv, group, tail):
    # 20 to 22 units: on both sides of the longest segment that blocks do not share; empty sequences between them
    rng = np.random.default_rng(kv * 10 + group)
    lengths = [20 * unit, 0, 21 * unit, 21 * unit + 1, 1, 0, 0, 22 * unit, 40 * unit, 3, 21 * unit - 1, 70, 0, tail]
    cache, q, pages, vals = attention_case(rng, len(lengths), kv, group, d, fmt, "bf16", lengths)
    lse = torch.empty(len(lengths), kv * group, dtype=torch.float32, device="cuda")
    out = cache.attend(q, ints(pages), ints(lengths), lse=lse)
    check_attention(cache, q, pages, lengths, vals, d ** -0.5, 0, out, lse, "bf16")
    again = cache.attend(q, ints(pages), ints(lengths))
    assert torch.equal(out, again)
    for b in range(len(lengths)):                # alone: other blocks, the same sums to rounding
        one = cache.attend(q[b:b + 1], ints(pages[b:b + 1]), ints(lengths[b:b + 1]))
        check_attention(cache, q[b:b + 1], pages[b:b + 1], lengths[b:b + 1], vals, d ** -0.5, 0, one, None, "bf16")


def test_attention_scores_far_apart_and_scale():
    # one key takes everything, its score hundreds above the others; then a scale of zero and a negative one
    rng = np.random.default_rng(13)
    cache, q, pages, vals = attention_case(rng, 2, 2, 4, 64, "bf16", "f32", [100, 37], spread=40.0)
    for scale in (1.0, 0.0, -0.5):
        lse = torch.empty(q.shape[:2], device="cuda")
        out = cache.attend(q, ints(pages), ints([100, 37]), scale=scale, lse=lse)
        check_attention(cache, q, pages, [100, 37], vals, scale, 0, out, lse, "f32")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_attention_with_scales_of_very_different_sizes(fmt):
    # V scales of a sequence differ by 2^40 and some heads are zero: small ones must not vanish beside each other's
    rng = np.random.default_rng(14)
    n = 90
    cache = PagedKV(1, 64, fmt, n_pages=6)
    mag = 2.0 ** rng.integers(-30, 10, n)
    mag[[3, 50]] = 0
    k, v = randn(rng, n, 1, 64), randn(rng, n, 1, 64) * torch.tensor(mag, device="cuda").float()[:, None, None]
    cache.append(k, v, ints(range(n)))
    kk, vv = (f64(t) for t in cache.read(ints(range(n)), dtype=torch.float32))
    q = randn(rng, 1, 3, 64)
    pages = np.arange(6)[None]
    out = cache.attend(q, ints(pages), ints([n]))
    vals = np.zeros((96, 2, 1, 64))
    vals[:n, 0], vals[:n, 1] = kk, vv
    check_attention(cache, q, pages, [n], vals, 0.125, 0, out, None, "f32")


def test_attention_of_a_nan_or_infinite_key_stays_in_its_sequence():
    rng = np.random.default_rng(15)
    lengths = [20, 20, 20]
    cache, q, pages, vals = attention_case(rng, 3, 1, 2, 64, "bf16", "f32", lengths)
    blocks = cache.data.view(torch.bfloat16).view(-1, 2, 1, 16, 64)
    blocks[int(pages[1][0]), 0, 0, 3, 10] = float("nan")
    blocks[int(pages[2][1]), 1, 0, 2, 10] = float("inf")
    out = cache.attend(q, ints(pages), ints(lengths))
    assert bool(torch.isnan(out[1]).all())
    assert not bool(torch.isfinite(out[2, :, 10]).any()) and bool(torch.isfinite(out[2, :, :10]).all())
    check_attention(cache, q[:1], pages[:1], lengths[:1], vals, 0.125, 0, out[:1], None, "f32")


def test_attention_strides_shared_pages_and_rows_past_the_batch():
    rng = np.random.default_rng(16)
    cache, _, pages, vals = attention_case(rng, 3, 2, 3, 64, "bf16", "bf16", [50, 64, 10])
    pages[2] = pages[0]                                        # a shared prefix
    big = randn(rng, 6, 7, 128, dtype="bf16")
    q = big[:6, :, :64].transpose(0, 1)[:3]                    # heads-first, strided rows
    out = torch.full((8, 9, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got = cache.attend(q, ints(pages), ints([50, 64, 10]), out=out[:, 1:7])
    check_attention(cache, q, pages, [50, 64, 10], vals, 0.125, 0, got, None, "bf16")
    assert bool((out[3:] == 7.0).all()) and bool((out[:, 0] == 7.0).all()) and bool((out[:, 7:] == 7.0).all())
    odd = torch.full((3 * 6 * 64 + 1,), 7.0, dtype=torch.bfloat16, device="cuda")[1:].view(3, 6, 64)
    qo = torch.empty(3 * 6 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(3, 6, 64)
    qo.copy_(q)                                                # 2-byte aligned
    cache.attend(qo, ints(pages), ints([50, 64, 10]), out=odd)
    assert torch.equal(odd, out[:3, 1:7])


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_bad_pages_and_lengths_give_nan_and_are_reported(fmt):
    rng = np.random.default_rng(17)
    lengths = [40, 40, 40, 40, 40]
    cache, q, pages, vals = attention_case(rng, 5, 2, 2, 64, fmt, "f32", lengths)
    pages[1, 2], pages[2, 0] = -1, cache.n_pages
    lse = torch.empty(q.shape[:2], device="cuda")
    out = cache.attend(q, ints(pages), ints(lengths), lse=lse)
    with pytest.raises(wici.WiciError, match="page"):
        cache.check()
    assert bool(torch.isnan(out[1:3]).all()) and bool(torch.isnan(lse[1:3]).all())
    for b in (0, 3, 4):
        check_attention(cache, q[b:b + 1], pages[b:b + 1], [40], vals, 0.125, 0, out[b:b + 1], lse[b:b + 1], "f32")
    out = cache.attend(q, ints(pages), ints([40, -5, -2 ** 31, 49, 2 ** 31 - 1]), lse=lse)
    with pytest.raises(wici.WiciError, match="length"):
        cache.check()
    assert bool((out[1:3] == 0).all()) and bool((lse[1:3] == -np.inf).all())
    assert bool(torch.isnan(out[3:]).all()) and bool(torch.isnan(lse[3:]).all())
    check_attention(cache, q[:1], pages[:1], [40], vals, 0.125, 0, out[:1], lse[:1], "f32")
    # a bad page before the window is not needed
    out = cache.attend(q, ints(pages), ints(lengths), window=9)
    with pytest.raises(wici.WiciError, match="page"):
        cache.check()
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isfinite(out[2]).all())


def test_attention_repeats_itself_and_workspaces_serve_any_order_of_calls():
    rng = np.random.default_rng(18)
    big, small = [3000, 10, 700], [30, 500, 0]
    cache, q, pages, _ = attention_case(rng, 3, 2, 4, 128, "int8", "bf16", [3000, 500, 700])
    ws = cache.workspace(8, 3)
    first = {}
    for i in range(6):
        for name, lengths in (("big", big), ("small", small)):
            out = cache.attend(q, ints(pages), ints(lengths), workspace=ws)
            assert torch.equal(out, first.setdefault(name, out)), (name, i)
    assert torch.equal(cache.attend(q, ints(pages), ints(big)), first["big"])
    with pytest.raises(ValueError, match="workspace"):
        cache.attend(q, ints(pages), ints(big), workspace=ws[:16])


def test_two_streams_at_once():
    rng = np.random.default_rng(19)
    lengths = [4000] * 4
    cache, q, pages, _ = attention_case(rng, 4, 2, 4, 64, "bf16", "bf16", lengths)
    p, n = ints(pages), ints(lengths)
    want = [cache.attend(q * (i + 1), p, n) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(cache.attend(q * (i + 1), p, n))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


# ----------------------------------------------------------------- together --
@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_a_decode_loop_of_a_batch_captured_and_replayed(fmt):
    """Prompts of several sequences appended at once, then decode steps (append + attend) as a captured graph whose
    inputs change between replays; every step against the oracle on what the cache then holds."""
    rng = np.random.default_rng(20)
    B, kv, group, d = 3, 2, 4, 64
    H = kv * group
    prompt, steps = [21, 0, 40], 12
    r = Rope(d, 1e4, scaling="bands", **SCALED["bands"])
    f, g = paged.rope_frequencies(d, 1e4, "bands", **SCALED["bands"])
    cache = PagedKV(kv, d, fmt, data=torch.full((12 * ops.wici_kv_page_bytes(ops.FORMATS[fmt], kv, d),), 255,
                                                dtype=torch.uint8, device="cuda"))
    pages = rng.permutation(12).reshape(B, 4)
    lengths = np.array(prompt)
    rows = randn(rng, sum(prompt), H + 2 * kv, d, dtype="bf16")
    pos = np.concatenate([np.arange(n) for n in prompt])
    seq = np.concatenate([np.full(n, b) for b, n in enumerate(prompt)])
    slots = pages[seq, pos // 16] * 16 + pos % 16
    cache.append(rows[:, H:H + kv], rows[:, H + kv:], ints(slots), rope=r, positions=ints(pos))

    step = torch.zeros(B, H + 2 * kv, d, dtype=torch.bfloat16, device="cuda")
    q_out, out = torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda")
    d_pos, d_slots, d_len, d_pages = ints([0] * B), ints([-1] * B), ints([0] * B), ints(pages)

    def one():
        cache.append(step[:, H:H + kv], step[:, H + kv:], d_slots, rope=r, positions=d_pos, q=step[:, :H], q_out=q_out)
        cache.attend(q_out, d_pages, d_len, out=out)

    before = cache.data.clone()
    one()                                                     # slots -1: nothing is written
    assert torch.equal(cache.data, before) and bool((out == 0).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for s in range(steps):
        live = np.array([True, True, s % 3 != 0])              # a client that pauses: padding
        step.copy_(randn(rng, B, H + 2 * kv, d, dtype="bf16"))
        slot = np.where(live, pages[np.arange(B), lengths // 16] * 16 + lengths % 16, -1)
        d_pos.copy_(ints(lengths))
        d_slots.copy_(ints(slot))
        now = lengths
        lengths = lengths + live
        d_len.copy_(ints(np.where(live, lengths, 0)))
        graph.replay()
        torch.cuda.synchronize()
        q64 = paged.rope(f64(step[:, :H]), now, d, f, g)
        mix = np.abs(f64(step[:, :H]))
        mix = np.tile(mix[..., :d // 2] + mix[..., d // 2:], 2)
        within(f64(q_out), q64, 2.0 ** -21 * g * mix + half_step(q64, "bf16"), "q")
        used = np.concatenate([pages[b, t // 16] * 16 + t % 16 for b in range(B) for t in [np.arange(lengths[b])]])
        vals = np.zeros((192, 2, kv, d))
        kk, vv = cache.read(ints(used), dtype=torch.float32)
        vals[used, 0], vals[used, 1] = f64(kk), f64(vv)
        check_attention(cache, q_out, pages, np.where(live, lengths, 0), vals, d ** -0.5, 0, out, None, "bf16")
    cache.check()


def test_two_captured_graphs_replayed_on_two_streams():
    rng = np.random.default_rng(21)
    lengths = [2500, 100, 1]
    cache, q, pages, _ = attention_case(rng, 3, 2, 4, 64, "e4m3", "f32", lengths)
    p, n = ints(pages), ints(lengths)
    want = cache.attend(q, p, n)
    outs, graphs = [torch.empty_like(q) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, o in zip(graphs, outs):
        with torch.cuda.graph(g):
            cache.attend(q, p, n, out=o)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        cache.attend(q, p, n)                                  # an eager call beside them
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_a_contexts_cache_read_attended_and_quantised():
    """A model's own cache through wici_kv_view: K and V of its prompt against the model oracle's, attention over it,
    and a batch of clients continuing from that prompt in an 8-bit cache."""
    cfg = gen.TINY
    w = gen.make_weights(cfg)
    prompt = gen.make_prompt(cfg, 45, seed=3)
    model = WiciModel(cfg, max_tokens=64).load(w)
    perm = np.random.default_rng(22).permutation(4)
    wici.wici_set_page_table(model.ctx, perm)
    model.prefill(prompt)
    ref = oracle.OracleModel(cfg, w, max_tokens=64)
    ref.prefill(prompt)
    kv, d = cfg.n_kv_heads, cfg.head_dim
    for layer in range(cfg.n_layers):
        k, v = model.read_kv(layer)
        assert k.shape == (45, kv, d)
        for got, want in ((k, ref.K[layer][:, :45]), (v, ref.V[layer][:, :45])):
            want = np.asarray(want, np.float64).transpose(1, 0, 2)
            err = np.linalg.norm(f64(got) - want) / np.linalg.norm(want)
            assert err <= 1e-2                                 # the model's own tolerance (bf16 storage is 1.7e-3 of it)
        part, _ = model.read_kv(layer, first=17, count=20)
        assert torch.equal(part, k[17:37])
        cache, table = model.kv_cache(layer)
        assert table.tolist() == perm.tolist()
        q = randn(np.random.default_rng(23), 1, cfg.n_q_heads, d)
        out = cache.attend(q, table[None], ints([45]))
        vals = np.zeros((64, 2, kv, d))
        order = perm[np.arange(45) // 16] * 16 + np.arange(45) % 16
        vals[order, 0], vals[order, 1] = f64(k), f64(v)
        check_attention(cache, q, perm[None], [45], vals, d ** -0.5, 0, out, None, "f32")
        small = PagedKV(kv, d, "int8", n_pages=3)
        small.append(k, v, ints(range(45)))
        k8, v8 = small.read(ints(range(45)), dtype=torch.float32)
        top = k.float().abs().amax(-1, keepdim=True)
        assert bool(((k8 - k.float()).abs() <= top * (0.5 / 127 + 2.0 ** -16)).all())
    with pytest.raises(wici.WiciError):
        model.kv_cache(cfg.n_layers)
    with pytest.raises(ValueError):
        model.read_kv(0, first=40, count=6)
    model.close()


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("group,d", [(9, 64), (16, 128), (33, 64)])
def test_attention_of_large_groups_in_fp32(fmt, group, d):
    # more than 8 queries to a KV head with more terms than a tile of 16 holds; odd counts leave a ragged last tile
    rng = np.random.default_rng(group)
    lengths = [130, 0, 61, 300]
    cache, q, pages, vals = attention_case(rng, 4, 2, group, d, fmt, "f32", lengths)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = cache.attend(q, ints(pages), ints(lengths), lse=lse, window=140)
    check_attention(cache, q, pages, lengths, vals, d ** -0.5, 140, out, lse, "f32")


@pytest.mark.parametrize("fmt,d", [("bf16", 64), ("bf16", 128), ("int8", 64), ("int8", 128), ("e4m3", 64), ("e4m3", 128)])
def test_attention_at_every_window_around_a_units_ends(fmt, d):
    # a unit is 1 to 4 pages: windows and lengths that begin and end in each of them
    rng = np.random.default_rng(24)
    lengths = list(range(60, 70)) + [128, 129, 1, 2]
    cache, q, pages, vals = attention_case(rng, len(lengths), 1, 2, d, fmt, "bf16", lengths)
    for window in (1, 15, 16, 17, 47, 48, 49, 63, 64, 65):
        out = cache.attend(q, ints(pages), ints(lengths), window=window)
        check_attention(cache, q, pages, lengths, vals, d ** -0.5, window, out, None, "bf16")


def test_equal_sequences_give_equal_results_wherever_their_runs_are_cut():
    # 40 sequences share one table row: the splits differ, the sums' order with them, the values only by rounding
    rng = np.random.default_rng(25)
    cache, q, pages, vals = attention_case(rng, 1, 2, 3, 64, "bf16", "f32", [777])
    out = cache.attend(q.expand(40, -1, -1).contiguous(), ints(np.repeat(pages, 40, 0)), ints([777] * 40))
    for b in (0, 1, 13, 39):
        check_attention(cache, q, pages, [777], vals, 0.125, 0, out[b:b + 1], None, "f32")
    assert bool(((out - out[:1]).abs() <= 2.0 ** -15).all())


def test_keys_whose_codes_are_small_beside_one_outlier():
    # a head whose scale one element sets: the other codes are 0 or 1, and an int8 score is the difference of larger sums
    rng = np.random.default_rng(26)
    n = 200
    x = rng.normal(size=(n, 1, 128))
    x[:, :, 5] = 100.0
    cache = PagedKV(1, 128, "int8", n_pages=13)
    cache.append(torch.tensor(x, device="cuda").float(), randn(rng, n, 1, 128), ints(range(n)))
    kk, vv = (f64(t) for t in cache.read(ints(range(n)), dtype=torch.float32))
    q = randn(rng, 1, 4, 128, dtype="bf16") + 1.0
    vals = np.zeros((208, 2, 1, 128))
    vals[:n, 0], vals[:n, 1] = kk, vv
    pages = np.arange(13)[None]
    out = cache.attend(q, ints(pages), ints([n]))
    # raised by 128, a score is off by up to 2 d 2^-23 of 128 sum |q| scale in place of sum |q k|
    want, _, weight = paged.paged_attention(f64(q), vals[:, 0], vals[:, 1], pages, [n], 128 ** -0.5)
    ds = 2 * 128 * 2.0 ** -23 * 128 * np.abs(f64(q)).sum(-1).max() * (100.0 / 127) * 128 ** -0.5
    within(f64(out), want, (2 * ds + 2.0 ** -16 + n * 2.0 ** -23) * weight + half_step(want, "bf16"), "outlier")


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_a_cache_of_more_than_4_gb(fmt):
    # byte offsets past 32 bits, in what is written, read and attended over
    rng = np.random.default_rng(27)
    kv, d, n = 8, 128, 100
    page = ops.wici_kv_page_bytes(ops.FORMATS[fmt], kv, d)
    pages = (1 << 32) // page + 5000
    cache = PagedKV(kv, d, fmt, data=torch.empty(pages * page, dtype=torch.uint8, device="cuda"))
    table = np.concatenate([[pages - 1, 3, pages - 2000], rng.permutation(4000)[:4] + pages - 4500])[None]
    slots = table[0, np.arange(n) // 16] * 16 + np.arange(n) % 16
    k, v = randn(rng, n, kv, d, dtype="bf16"), randn(rng, n, kv, d, dtype="bf16")
    cache.append(k, v, ints(slots))
    kk, vv = cache.read(ints(slots), dtype=torch.float32)
    top = torch.stack([k, v]).float().abs().amax(-1, keepdim=True)
    err = (torch.stack([kk, vv]) - torch.stack([k, v]).float()).abs()
    assert bool((err <= (0 if fmt == "bf16" else (0.5 / 127 + 2.0 ** -16)) * top).all())
    q = randn(rng, 1, 16, d)
    out = cache.attend(q, ints(table), ints([n]))
    cache.check()
    vals = np.zeros((16 * 7, 2, kv, d))
    vals[:n, 0], vals[:n, 1] = f64(kk), f64(vv)
    check_attention(cache, q, np.arange(7)[None], [n], vals, d ** -0.5, 0, out, None, "f32")


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_pages_of_several_layers_side_by_side(fmt):
    # page_stride: [page][layer] pools, one layer of which is this cache; the other layers' bytes stay
    rng = np.random.default_rng(28)
    kv, d, layers, pages, n = 3, 64, 3, 5, 70
    page = ops.wici_kv_page_bytes(ops.FORMATS[fmt], kv, d)
    pool = torch.full((pages, layers, page), 255, dtype=torch.uint8, device="cuda")
    cache = ops.wici_kv_cache(pool[0, 1].data_ptr(), layers * page, pages, kv, d, ops.FORMATS[fmt])
    plain = PagedKV(kv, d, fmt, data=torch.full((pages * page,), 255, dtype=torch.uint8, device="cuda"))
    k, v, q = (randn(rng, n, kv, d), randn(rng, n, kv, d), randn(rng, 1, 6, d))
    table, st = rng.permutation(pages)[None], torch.cuda.current_stream().cuda_stream
    slots, dev = ints(table[0, np.arange(n) // 16] * 16 + np.arange(n) % 16), k.device
    hk, hv = ops.heads_of(k, d, dev, "k"), ops.heads_of(v, d, dev, "v")
    ops.wici_kv_append(st, cache, slots.data_ptr(), n, hk, hv)
    plain.append(k, v, slots)
    assert torch.equal(pool[:, 1].reshape(-1), plain.data)
    assert bool((pool[:, 0] == 255).all()) and bool((pool[:, 2] == 255).all())
    back = [torch.empty(n, kv, d, device="cuda") for _ in range(2)]
    ops.wici_kv_read(st, cache, slots.data_ptr(), n, *(ops.heads_of(b, d, dev, "b") for b in back))
    assert all(torch.equal(a, b) for a, b in zip(back, plain.read(slots, dtype=torch.float32)))
    out, ws = torch.empty_like(q), plain.workspace(6, 1)
    p, length = ints(table), ints([n])
    ops.wici_paged_attention(st, cache, ops.wici_attn_shape(1, pages, 0, 0.125), p.data_ptr(), length.data_ptr(),
                             ops.heads_of(q, d, dev, "q"), ops.heads_of(out, d, dev, "o"), None, ws.data_ptr())
    assert torch.equal(out, plain.attend(q, p, length, scale=0.125))


def test_broadcast_keys_and_odd_alignments_take_the_narrow_path_to_the_same_bytes():
    rng = np.random.default_rng(29)
    T, kv, d = 21, 4, 64
    rope = Rope(d, 1e4, rot_dim=32)
    slots, pos = ints(rng.permutation(32)[:T]), ints(rng.integers(0, 9999, T))
    base = randn(rng, T, 1, d, dtype="bf16")
    k, v = base.expand(T, kv, d), randn(rng, T, kv, d, dtype="bf16")
    q = randn(rng, T, 5, d, dtype="bf16")

    def odd(x):                                                # the same values, 2-byte aligned
        y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        return y.copy_(x)

    for fmt in ("bf16", "int8", "e4m3"):
        a, b = PagedKV(kv, d, fmt, n_pages=2), PagedKV(kv, d, fmt, n_pages=2)
        qa = a.append(k.contiguous(), v, slots, rope=rope, positions=pos, q=q)
        qb = b.append(odd(k), odd(v), slots, rope=rope, positions=pos, q=odd(q), q_out=odd(q))
        assert torch.equal(a.data, b.data) and torch.equal(qa, qb)
        b.data.zero_()
        b.append(k, v, slots, rope=rope, positions=pos)        # heads of stride 0, and no q
        assert torch.equal(a.data, b.data)


@pytest.mark.parametrize("fmt,group,batch", [("bf16", 1, 2100), ("int8", 9, 600)])
def test_batches_of_more_sequences_than_a_launch_takes(fmt, group, batch):
    rng = np.random.default_rng(30)
    lengths = rng.integers(-1, 36, batch)
    lengths[[0, 255, 256, 512, 599, batch - 1]] = [0, 17, 33, 0, 1, 20]
    cache, q, pages, vals = attention_case(rng, batch, 1, group, 64, fmt, "bf16", lengths)
    out, lse = torch.full((batch + 2, group, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.empty(batch, group, device="cuda")
    cache.attend(q, ints(pages), ints(lengths), out=out, lse=lse)
    cache.check()
    check_attention(cache, q, pages, lengths, vals, 0.125, 0, out, lse, "bf16")
    assert bool((out[batch:] == 7.0).all())


# token counts on both sides of what changes the tokens of a block (1, 2, 4 and 8 of them with 152 SMs), most of them ragged
LONG = [4863, 4864, 9729, 19457]


@pytest.mark.parametrize("tokens", LONG)
@pytest.mark.parametrize("dtype,d,rot,interleaved,odd", [
    ("bf16", 128, 128, False, False), ("f32", 64, 32, False, False), ("f16", 96, 64, True, False), ("bf16", 128, 126, False, False),
    ("bf16", 256, 100, False, True), ("f32", 256, 254, False, True), ("f16", 244, 18, False, False),
])
def test_rope_of_many_tokens(tokens, dtype, d, rot, interleaved, odd):
    # wide, ragged and element-wise paths; heads of up to 17 lanes
    rng = np.random.default_rng(tokens + d)
    pos = rng.integers(-3, 1 << 20, tokens)
    x = randn(rng, tokens * 3 * d + 1, dtype=dtype)[1 if odd else 0:][:tokens * 3 * d].view(tokens, 3, d)
    y = torch.full((tokens + 1, 3, d), 7.0, dtype=DT[dtype], device="cuda")
    Rope(d, 5e5, rot_dim=rot, interleaved=interleaved).apply(x, ints(pos), out=y[:tokens])
    check_rope(x, y[:tokens], pos, rot, 5e5, interleaved, "none", False, dtype)
    assert bool((y[tokens] == 7.0).all())


def check_stored(codes, scales, slots, which, x, fmt, turned):
    """K (which 0) or V of a cache at slots against x, in 64 bits.  A rotated element is off by up to 2^-21 (|x_a| + |x_b|),
    and |x_a| + |x_b| <= 2 amax of the rotated head: 2^-20 amax, however small the element itself has become.  So a
    quotient is off by top 2^-20, top the largest code, by as much of the scale's own error, and by 2^-22 of itself:
    below top 2^-18; one of given values by top 2^-22."""
    live = slots >= 0
    x, got = x[live], codes[slots[live], which]
    amax = np.abs(x).max(-1, keepdims=True)
    if fmt == "bf16":
        val = (got.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
        return within(val, x, half_step(x, "bf16") + (2.0 ** -20 * amax if turned else 0), "bf16 cache")
    top = 127.0 if fmt == "int8" else 448.0
    grid = np.arange(128.0) if fmt == "int8" else paged.E4M3[:127]
    s = scales[slots[live], which]
    within(s, amax[..., 0] / top, amax[..., 0] / top * (2.0 ** -19 if turned else 2.0 ** -23), "scale")
    gv, q, near = np.abs(paged.code_values(got, fmt)), np.abs(x) * top / amax, top * 2.0 ** (-18 if turned else -22)
    at = np.searchsorted(grid, gv)                             # the quotients that may round to this code, and `near` of them
    lo = np.where(at > 0, (grid[np.maximum(at - 1, 0)] + gv) / 2, 0.0)
    hi = np.where(at < grid.size - 1, (grid[np.minimum(at + 1, grid.size - 1)] + gv) / 2, top)
    assert np.all(grid[at] == gv) and np.all((q >= lo - near) & (q <= hi + near)), f"{fmt} codes"
    assert np.all((paged.code_values(got, fmt) * x >= 0) | (q <= near)), f"{fmt} signs"


@pytest.mark.parametrize("tokens", LONG)
@pytest.mark.parametrize("fmt,dtype,d", [("bf16", "bf16", 64), ("int8", "f32", 128), ("e4m3", "f16", 64), ("e4m3", "bf16", 128)])
def test_append_and_read_of_many_tokens(fmt, dtype, d, tokens):
    rng = np.random.default_rng(tokens + d)
    pages, kv, q_heads = tokens // 16 + 3, 2, 3
    before = torch.tensor(rng.integers(0, 256, pages * ops.wici_kv_page_bytes(ops.FORMATS[fmt], kv, d)), dtype=torch.uint8,
                          device="cuda")
    cache = PagedKV(kv, d, fmt, data=before.clone())
    k, v, q = (randn(rng, tokens, n, d, dtype=dtype) for n in (kv, kv, q_heads))
    slots, pos = slots_for(rng, tokens, pages), rng.integers(0, 100000, tokens)
    slots[[3, tokens - 1]] = [-1, -7]
    r, (f, g) = Rope(d, 5e5), paged.rope_frequencies(d, 5e5)
    q_out = cache.append(k, v, ints(slots), rope=r, positions=ints(pos), q=q)
    cache.check()
    check_rope(q, q_out, pos, d, 5e5, False, "none", False, dtype)
    codes, scales = paged.unpack(cache.data.cpu().numpy(), kv, d, fmt)
    others = np.ones(pages * 16, bool)
    others[slots[slots >= 0]] = False
    for now, was in zip((codes, scales), paged.unpack(before.cpu().numpy(), kv, d, fmt)):
        assert now is None or np.array_equal(now[others].view(np.uint8), was[others].view(np.uint8))
    check_stored(codes, scales, slots, 0, paged.rope(f64(k), pos, d, f, g), fmt, True)
    check_stored(codes, scales, slots, 1, f64(v), fmt, False)
    got = cache.read(ints(slots), dtype=DT[dtype])
    for which in (0, 1):
        c = codes[slots, which]
        want = (c.astype(np.uint32) << 16).view(np.float32).astype(np.float64) if fmt == "bf16" else \
            paged.code_values(c, fmt) * scales[slots, which][..., None].astype(np.float64)
        want[slots < 0] = 0
        within(f64(got[which]), want, half_step(want, dtype) + 2.0 ** -24 * np.abs(want), "read")


def model_on_a_stream_of_its_own():
    cfg = gen.TINY
    model = WiciModel(cfg, max_tokens=64, stream=torch.cuda.Stream()).load(gen.make_weights(cfg))
    model.prefill(gen.make_prompt(cfg, 45, seed=3))
    return model


def test_what_read_kv_gives_outlives_the_next_read_on_the_callers_stream():
    # a caller on another stream than the context's drops a layer's K and V with its own work on them still queued
    model = model_on_a_stream_of_its_own()
    layers = range(model.cfg.n_layers)
    want = [[t.clone() for t in model.read_kv(i)] for i in layers]
    torch.cuda.synchronize()
    small = [PagedKV(model.cfg.n_kv_heads, model.cfg.head_dim, "bf16", n_pages=3) for _ in layers]
    slots = ints(range(45))
    for _ in range(3):
        torch.cuda._sleep(20_000_000)                         # about 10 ms: the reads below run ahead of this stream
        for i in layers:
            k, v = model.read_kv(i)
            small[i].append(k, v, slots)
            del k, v
        torch.cuda.synchronize()
        for i in layers:
            assert all(torch.equal(a, b) for a, b in zip(small[i].read(slots), want[i])), i
            small[i].data.zero_()
    model.close()


def test_a_contexts_cache_reports_calls_on_its_stream_whatever_the_callers_does():
    model = model_on_a_stream_of_its_own()
    bad = ints([1 << 20])
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                             # the caller's stream is behind the context's
    cache, _ = model.kv_cache(0)
    with torch.cuda.stream(model.stream):
        cache.read(bad)
    torch.cuda.synchronize()
    with pytest.raises(wici.WiciError, match="slot"):
        cache.check()
    model.close()


@pytest.mark.parametrize("group", [4, 12])
def test_scores_of_small_int8_codes_keep_their_bits(group):
    # one channel sets the scales of the keys, and the queries do not look at it: the codes that they meet are 0 to 4; a
    # second one is large in the queries and zero in the keys.
    # A score's products are exact in fp32, and each of its d sums drops at most 2^-23 of sum |q k| (tensor cores may
    # truncate): d 2^-23 sum |q k|, not of what the codes' whole range would allow.
    rng = np.random.default_rng(31)
    n, d = 40, 64
    x = 10 * rng.normal(size=(n, 1, d))
    x[:, :, 5], x[:, :, 7] = 1000.0, 0.0
    cache = PagedKV(1, d, "int8", n_pages=3)
    cache.append(torch.tensor(x, device="cuda").float(), randn(rng, n, 1, d), ints(range(n)))
    kk, vv = (f64(t)[:, 0] for t in cache.read(ints(range(n)), dtype=torch.float32))
    q = 1 + 0.1 * randn(rng, 1, group, d)
    q[:, :, 5], q[:, :, 7] = 0.0, 3000.0
    q = q.to(torch.bfloat16)
    lse, out = torch.empty(1, group, device="cuda"), torch.empty(1, group, d, device="cuda")
    cache.attend(q, ints([[0, 1, 2]]), ints([n]), lse=lse, out=out)
    s = f64(q)[0] @ kk.T * d ** -0.5
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    want_lse = (top + np.log(p.sum(-1, keepdims=True)))[:, 0]
    p /= p.sum(-1, keepdims=True)
    ds = d * 2.0 ** -23 * (np.abs(f64(q)[0]) @ np.abs(kk).T).max(-1) * d ** -0.5 + 2.0 ** -23 * np.abs(s).max(-1)
    # the exponential to 2^-21, a sum of n to n 2^-23, the logarithm and lse's own rounding
    rest = 2.0 ** -21 + n * 2.0 ** -23
    within(f64(lse)[0], want_lse, ds + rest + 2.0 ** -22 * np.abs(want_lse), "lse")
    within(f64(out)[0], p @ vv, (2 * ds + 2 * rest + 2.0 ** -21)[:, None] * (p @ np.abs(vv)) + 2.0 ** -24 * np.abs(p @ vv), "out")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,group,n", [("bf16", 4, 300), ("f32", 3, 300), ("bf16", 12, 300), ("bf16", 2, 5000)])
@pytest.mark.parametrize("shift,score", [(20, -70.0), (34, -70.0), (60, -80.0), (-40, 20.0), (-40, 45.0), (100, -75.0)])
def test_one_key_whose_v_is_of_another_size_than_the_others(fmt, dtype, group, n, shift, score):
    # one key's V is 2^shift times the others', its score `score` above theirs: large values that hardly count, or a key
    # that takes most of the weight with next to no value.  The result is held to sum p |v|, wherever the key stands.
    rng = np.random.default_rng(32)
    d = 64
    k, v = 0.05 * rng.normal(size=(n, 1, d)), rng.normal(size=(n, 1, d)) + 0.5
    q = 0.2 * rng.normal(size=(1, group, d))
    q[..., 9], k[..., 9] = 4.0, 0.0
    for at in (0, 16 * 7 + 3, n - 1):
        kk, vv = k.copy(), v.copy()
        kk[at, 0, 9], vv[at] = score / 4.0, v[at] * 2.0 ** shift
        cache = PagedKV(1, d, fmt, n_pages=(n + 15) // 16)
        cache.append(torch.tensor(kk, device="cuda").float(), torch.tensor(vv, device="cuda").float(), ints(range(n)))
        stored = [f64(t) for t in cache.read(ints(range(n)), dtype=torch.float32)]
        qq = torch.tensor(q, device="cuda").to(DT[dtype])
        pages, vals = np.arange(cache.n_pages)[None], np.zeros((cache.n_pages * 16, 2, 1, d))
        vals[:n, 0], vals[:n, 1] = stored
        lse, out = torch.empty(1, group, device="cuda"), torch.empty(1, group, d, device="cuda")
        cache.attend(qq, ints(pages), ints([n]), scale=1.0, lse=lse, out=out)
        check_attention(cache, qq, pages, [n], vals, 1.0, 0, out, lse, dtype, "f32")


@pytest.mark.parametrize("dtype,group", [("bf16", 4), ("f32", 4), ("f16", 12), ("bf16", 12)])
def test_infinite_keys_and_values_follow_the_formula(dtype, group):
    # a weight times an infinite value is that infinity, two of them NaN; a key whose score is -infinity has no weight,
    # one of +infinity makes NaN; the rest of the sequence's result, and the other sequences', as if nothing were there
    rng = np.random.default_rng(33)
    d, kv, lengths = 64, 2, [20, 40, 40, 600]
    cache, q, pages, vals = attention_case(rng, 4, kv, group, d, "bf16", dtype, lengths)
    q[:, :, 10] = q[:, :, 10].abs() + 0.25
    q[3, 1, 10] *= -1
    blocks, inf = cache.data.view(torch.bfloat16).view(-1, 2, kv, 16, d), float("inf")

    def put(b, t, which, head, i, x):
        page = int(pages[b][t // 16])
        blocks[page, which, head, t % 16, i] = x
        vals[page * 16 + t % 16, which, head, i] = x

    put(1, 3, 1, 0, 10, inf)
    put(1, 33, 1, 0, 11, -inf)
    put(1, 4, 1, 1, 12, inf), put(1, 37, 1, 1, 12, -inf)
    put(2, 5, 0, 0, 10, -inf)                                 # no weight
    put(2, 17, 0, 1, 10, inf)                                 # NaN
    put(3, 500, 0, 0, 10, -inf)                               # no weight; for the query of the other sign NaN
    put(3, 599, 1, 1, 63, inf), put(3, 0, 1, 1, 63, inf)
    lse, out = torch.empty(4, kv * group, device="cuda"), torch.empty(4, kv * group, d, device="cuda")
    cache.attend(q, ints(pages), ints(lengths), lse=lse, out=out)
    for b, n in enumerate(lengths):
        slots = [int(pages[b][t // 16]) * 16 + t % 16 for t in range(n)]
        for h in range(kv * group):
            k, v, q64 = vals[slots, 0, h // group], vals[slots, 1, h // group], f64(q)[b, h]
            with np.errstate(invalid="ignore"):
                s = k @ q64 * d ** -0.5
                p = np.exp(s - s.max())
                want, got = p @ v / p.sum(), f64(out)[b, h]
                want_lse = s.max() + np.log(p.sum())
            if np.isnan(want_lse):
                assert np.isnan(got).all() and np.isnan(float(lse[b, h]))
                continue
            assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(want[np.isinf(want)], got[np.isinf(want)])
            there = np.isfinite(s)                            # of the keys that count
            size = (np.abs(k[there]) @ np.abs(q64)).max() * d ** -0.5
            ds = size * (2 * d * 2.0 ** -23 + (2.0 ** -16 if dtype == "f32" else 0.0))
            weight = p[there] @ np.where(np.isfinite(v[there]), np.abs(v[there]), 0) / p.sum()
            fine = np.isfinite(want)
            within(got[fine], want[fine], ((2 * ds + 2.0 ** -16 + 2.0 ** -21 + n * 2.0 ** -23) * weight)[fine] + 1e-30, f"sequence {b}, head {h}")
            within(float(lse[b, h]), want_lse, ds + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -23 * abs(want_lse), "lse")


def test_a_stream_keeps_one_workspace_for_every_batch_and_head_count(monkeypatch):
    rng = np.random.default_rng(34)
    cache, _, pages, vals = attention_case(rng, 6, 2, 1, 64, "bf16", "bf16", [40, 1, 0, 700, 33, 16])
    lengths, made, make = [40, 1, 0, 700, 33, 16], [], cache.workspace
    monkeypatch.setattr(cache, "workspace", lambda *a: made.append(a) or make(*a))
    other = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), other):
        for batch, group in ((1, 1), (2, 1), (6, 1), (3, 5), (6, 16), (1, 16), (6, 1)):
            q = randn(rng, batch, 2 * group, 64, dtype="bf16")
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                out = cache.attend(q, ints(pages[:batch]), ints(lengths[:batch]))
            torch.cuda.synchronize()
            check_attention(cache, q, pages[:batch], lengths[:batch], vals, 0.125, 0, out, None, "bf16")
    assert len(made) == 2


@pytest.mark.parametrize("dtype,rot,interleaved,scaling", [("f32", 24, True, "yarn"), ("bf16", 32, False, "none"), ("f32", 32, False, "bands")])
@pytest.mark.parametrize("inverse", [False, True])
def test_autograd_sees_a_rotation(dtype, rot, interleaved, scaling, inverse):
    rng = np.random.default_rng(35)
    T, H, d = 5, 3, 32
    r = Rope(d, 1e4, rot_dim=rot, interleaved=interleaved, scaling=scaling, **SCALED[scaling])
    f, g = paged.rope_frequencies(rot, 1e4, scaling, **SCALED[scaling])
    pos = rng.integers(0, 3000, T)
    x, w = randn(rng, T, H, d, dtype=dtype).requires_grad_(), randn(rng, T, H, d, dtype=dtype)
    y = r.apply(x, ints(pos), inverse=inverse)
    with torch.no_grad():
        assert torch.equal(y, r.apply(x, ints(pos), inverse=inverse)) and not r.apply(x, ints(pos)).requires_grad
    dx, = torch.autograd.grad(y, x, w)
    check_rope(w, dx, pos, rot, 1e4, interleaved, scaling, not inverse, dtype)           # the formula's gradient
    if dtype == "f32":                                        # and that of differences: the map is linear, the step is 1
        for i in range(0, d, 5):
            e = np.zeros((1, 1, d))
            e[..., i] = 0.5
            up, down = (paged.rope(f64(x) + s * e, pos, rot, f, g, interleaved, inverse) for s in (1, -1))
            # off by 2^-21 (|w_a| + |w_b|) g, at most 2^-20 g max |w|, and half a step
            within(f64(dx)[..., i], (f64(w) * (up - down)).sum(-1), 2.0 ** -19 * g * float(w.abs().max()), "differences")


def test_gradients_of_rotations_of_broadcast_heads_and_of_gradients():
    rng = np.random.default_rng(36)
    T, H, d = 4, 6, 64
    r, pos = Rope(d, 1e4), ints(rng.integers(0, 999, T))
    one = randn(rng, T, 1, d).requires_grad_()
    w = randn(rng, T, H, d)
    dx, = torch.autograd.grad(r.apply(one.expand(T, H, d), pos), one, w)
    back = r.apply(w, pos, inverse=True)
    within(f64(dx), f64(back).sum(1, keepdims=True), H * 2.0 ** -23 * np.abs(f64(back)).sum(1, keepdims=True), "shared heads")
    x = randn(rng, T, H, d).requires_grad_()
    r.apply(x, pos).sum().backward()                          # a gradient whose elements share one place
    assert torch.equal(x.grad, r.apply(torch.ones_like(w), pos, inverse=True))
    v = randn(rng, T, H, d).requires_grad_()
    dx, = torch.autograd.grad(r.apply(x, pos), x, v, create_graph=True)
    dv, = torch.autograd.grad(dx, v, w)                       # the gradient's own gradient: forward again
    assert torch.equal(dv, r.apply(w, pos))
    with pytest.raises(ValueError):
        r.apply(x, pos[:3])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,group", [("bf16", 4), ("f32", 5), ("f16", 12)])
def test_weights_far_below_the_heaviest(fmt, dtype, group):
    # scores tens apart: where the heaviest key's code is 0, what is left of an element are weights of 2^-20 and less.  A
    # weight times its scale is in fp16 terms whose last half bit, 2^-25, is 2^-32 of the heaviest (at least 2^7 of those
    # units): each code adds that much of its own size to the tolerance on sum p |v|.
    rng = np.random.default_rng(37)
    lengths, d, kv = [12, 90, 333, 3], 64, 2
    cache, q, pages, vals = attention_case(rng, 4, kv, group, d, fmt, dtype, lengths)
    out = torch.empty(q.shape, device="cuda")
    cache.attend(q, ints(pages), ints(lengths), scale=1.0, out=out)
    q64 = f64(q)
    want, _, weight = paged.paged_attention(q64, vals[:, 0], vals[:, 1], pages, lengths, 1.0, 0)
    for b, n in enumerate(lengths):
        slots = [int(pages[b][t // 16]) * 16 + t % 16 for t in range(n)]
        for h in range(q.shape[1]):
            k, v = vals[slots, 0, h // group], vals[slots, 1, h // group]
            p = np.exp(k @ q64[b, h] - (k @ q64[b, h]).max())
            scale = np.abs(v).max(-1, keepdims=True) / (127 if fmt == "int8" else 448)    # every head's largest code is the top one
            floor = 2.0 ** -32 * (p * scale[:, 0]).max() / p.sum() * np.abs(v / scale).sum(0)
            ds = float(np.max(np.abs(k) @ np.abs(q64[b, h]))) * (2 * d * 2.0 ** -23 + (2.0 ** -16 if dtype == "f32" else 0.0))
            within(f64(out)[b, h], want[b, h], (2 * ds + 2.0 ** -16 + 2.0 ** -21 + n * 2.0 ** -23) * weight[b, h] + floor,
                   f"sequence {b}, head {h}")


@pytest.mark.parametrize("dtype,d,tokens", [("bf16", 128, 700), ("f16", 64, 700), ("f32", 64, 300), ("bf16", 64, 5000)])
def test_int8_codes_are_the_nearest_to_the_quotient_itself(dtype, d, tokens):
    # many quotients of 16-bit values are ties of x 127 / max; of x / scale, whose scale is rounded to fp32, they lie up to
    # 2^-25 beside the border, and nearer than that never, so 64 bits tell the side: codes are compared exactly
    rng = np.random.default_rng(38)
    pages = tokens // 16 + 1
    cache = PagedKV(2, d, "int8", n_pages=pages)
    k, v = randn(rng, tokens, 2, d, dtype=dtype), randn(rng, tokens, 2, d, dtype=dtype)
    v[:, 0] = (127 * v[:, 0].float()).round().to(DT[dtype]) * 0.5
    v[:, 0, 0] = 127.0 if dtype != "bf16" else 254.0           # a scale of 1 or 2: true ties, to the even code
    v[:, 0].clamp_(-127.0 if dtype != "bf16" else -254.0, float(v[0, 0, 0]))
    v[5] *= 2.0 ** (-12 if dtype == "f16" else -116)           # scales near the end of the normal range
    slots = slots_for(rng, tokens, pages)
    cache.append(k, v, ints(slots))
    codes, scales = paged.unpack(cache.data.cpu().numpy(), 2, d, "int8")
    for which, x in ((0, f64(k)), (1, f64(v))):
        s = scales[slots, which]
        np.testing.assert_array_equal(s, (np.abs(x).max(-1).astype(np.float32) / np.float32(127)))
        keep = s >= 2.0 ** -126
        q = x / np.where(keep, s, 1).astype(np.float64)[..., None]
        np.testing.assert_array_equal(codes[slots, which].view(np.int8)[keep], np.rint(q)[keep])
