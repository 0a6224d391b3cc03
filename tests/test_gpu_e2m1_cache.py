"""The 4-bit cache format (e2m1 codes, e4m3 block scales, fp32 scales) of a batched decode step's operators through
their binding, against the fp64 oracle (oracle/paged.py).

Tolerances as in tests/test_gpu_ops.py; of the format itself:
* codes and block scales of given values are decided exactly, scales are one fp32 division: nothing differs but a scale's
  last place where the oracle's double quotient was rounded twice (2^-23 of it).
* rotated values are off by 2^-21 (|x_a| + |x_b|) g <= 2^-20 * 1.42 g max|x|, as is the scale.  The unit b s of a block
  is the stored one, so a value's distance to its code exceeds the nearest code's by twice that at most.
* read values: code * b is exact, its product with the scale is rounded to fp32 (2^-24), then to the type.
"""
import numpy as np
import pytest

from oracle import paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2608_24204_gb300 import PagedKV, Rope, ops, wici  # noqa: E402
from tests.test_gpu_ops import DT, SCALED, check_attention, check_rope, f64, half_step, ints, randn, slots_for, within  # noqa: E402


def values(c):
    return np.where(c == 8, 0, c)                               # -0 is 0


def check_stored(data, before, slots, k, v, kv, d, turned, g=1.0):
    got, old = paged.unpack_e2m1(data.cpu().numpy(), kv, d), paged.unpack_e2m1(before.cpu().numpy(), kv, d)
    live = slots >= 0
    others = np.ones(got[0].shape[0], bool)
    others[slots[live]] = False
    for a, b in zip(got, old):
        np.testing.assert_array_equal(a[others].view(np.uint8), b[others].view(np.uint8))
    for which, x in ((0, k), (1, v)):
        codes, each, scales = (a[slots[live], which] for a in got)
        x = x[live]
        if not (turned and which == 0):
            want = paged.quantise_e2m1(x)
            within(scales, want[2], want[2] * 2.0 ** -23, "scale")
            same = (scales == want[2])[..., None]
            # a scale that is off in its last place has quotients of its own
            assert np.all((each == want[1]) | ~same) and np.all((values(codes) == values(want[0])) | ~same)
            assert same.mean() > 0.99
            continue
        top = np.abs(x).max(-1)
        off = 2.0 ** -20 * 1.42 * g * top
        within(scales, top / 2688, off / 2688 + 2.0 ** -23 * top / 2688, "scale of rotated keys")
        s = scales.astype(np.float64)
        block = np.abs(x).reshape(*x.shape[:-1], -1, 16).max(-1)
        b = paged.E4M3[each]
        y = np.where(s[..., None] > 0, block / (6 * np.where(s > 0, s, 1)[..., None]), 0)
        best = paged.E4M3[paged.e4m3_codes(y)]
        assert np.all(np.abs(y - b) <= np.abs(y - best) + 2 * 448 * 2.0 ** -19 * 1.42 * g)
        unit = b * s[..., None]
        err = np.abs(x - paged.e2m1_values(codes, each, scales)).reshape(*unit.shape, 16)
        xs = np.abs(x).reshape(*unit.shape, 16)
        gap = np.abs(xs[..., None] - paged.E2M1[:8] * unit[..., None, None]).min(-1)
        assert np.all(err <= gap + 2 * off[..., None, None])


@pytest.mark.parametrize("dtype,tokens,kv,d,q_heads,rot,scaling,interleaved", [
    ("bf16", 1, 8, 128, 32, 128, "bands", False),
    ("f32", 1, 1, 64, 0, 0, "none", False),
    ("f16", 17, 2, 64, 6, 64, "none", True),
    ("bf16", 100, 3, 128, 15, 48, "yarn", False),    # halves of 24: blocks of two lanes' first and second groups
    ("f32", 333, 8, 128, 8, 128, "linear", False),
    ("f16", 50, 5, 128, 0, 0, "none", False),
    ("bf16", 1000, 4, 64, 0, 16, "none", False),
    ("f32", 40, 2, 128, 3, 80, "none", False),
    ("f16", 5000, 1, 64, 2, 32, "none", True),
    ("bf16", 9000, 2, 128, 0, 0, "none", False),
])
def test_append_and_read(dtype, tokens, kv, d, q_heads, rot, scaling, interleaved):
    rng = np.random.default_rng(tokens + d)
    pages = tokens // 16 + 3
    before = torch.tensor(rng.integers(0, 256, pages * ops.wici_kv_page_bytes(ops.WICI_KV_E2M1, kv, d)), dtype=torch.uint8, device="cuda")
    cache = PagedKV(kv, d, "e2m1", data=before.clone())
    k, v = randn(rng, tokens, kv, d, dtype=dtype, scale=3.0), randn(rng, tokens, kv, d, dtype=dtype)
    if tokens > 3:
        v[1] = 0                                              # a head of zeros
        v[2, :, 16:32] = 0                                    # a block of zeros
        k[2, 0] *= 2.0 ** -10
        k[0, :, :16] *= 2.0 ** -12                            # a block far below the others
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
    check_stored(cache.data, before, slots, k64, f64(v), kv, d, bool(rot), g)
    if q_heads:
        check_rope(kw["q"], q_out, pos, rot, 5e5, interleaved, scaling, False, dtype)
    stored = paged.unpack_e2m1(cache.data.cpu().numpy(), kv, d)
    back = np.concatenate([slots[::-1], slots[:2], [-3]])     # any order, repeats, padding
    for out_dtype in DT:
        got = cache.read(ints(back), dtype=DT[out_dtype])
        for which in (0, 1):
            want = paged.e2m1_values(*(a[back, which] for a in stored))
            want[back < 0] = 0
            within(f64(got[which]), want, half_step(want, out_dtype) + 2.0 ** -24 * np.abs(want), f"read {out_dtype}")


@pytest.mark.parametrize("dtype,d,shift", [("bf16", 128, 0), ("f16", 64, 0), ("bf16", 64, 0), ("f32", 64, 0), ("f32", 128, -60), ("bf16", 64, 100)])
def test_codes_of_values_half_way_between_codes(dtype, d, shift):
    """Values built on the middles between codes, of blocks whose scales are exact or next to a middle themselves."""
    rng = np.random.default_rng(d + shift)
    tokens = 600
    unit = 2.0 ** shift * np.array([1.0, 7.0, 1.75, 3.5])[rng.integers(0, 4, tokens)]
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, 1.5])
    x = grid[rng.integers(0, len(grid), (tokens, 1, d))] * rng.choice([-1.0, 1.0], (tokens, 1, d))
    x[:, :, 0] = 6.0
    x = x.reshape(tokens, 1, -1, 16) * 2.0 ** -rng.integers(0, 6, (tokens, 1, d // 16, 1)) * rng.choice([1.0, 1.0625, 1.125], (tokens, 1, d // 16, 1))
    x[:, :, 0] *= 64.0
    x = x.reshape(tokens, 1, d) * unit[:, None, None]
    t = torch.tensor(x, device="cuda").to(DT[dtype])
    if dtype == "f32":                                        # and the neighbours of the middles
        t = torch.where(torch.tensor(rng.random(t.shape) < 0.3, device="cuda"), torch.nextafter(t, t * 2), t)
    cache = PagedKV(1, d, "e2m1", n_pages=tokens // 16 + 1)
    before = cache.data.clone()
    slots = np.arange(tokens)
    cache.append(t, -t, ints(slots))
    check_stored(cache.data, before, slots, f64(t), -f64(t), 1, d, False)


def test_append_of_infinities_nans_and_tiny_heads():
    k = torch.ones(6, 1, 64, device="cuda")
    k[0, 0, 5], k[1, 0, 63], k[2] = float("inf"), float("nan"), 1e-40
    k[3] = 1e-25
    k[5, 0, ::2] = 3e38                                       # the largest scales
    cache = PagedKV(1, 64, "e2m1", n_pages=1)
    cache.append(k, -k, ints(range(6)))
    kk, vv = (f64(t)[:, 0] for t in cache.read(ints(range(6)), dtype=torch.float32))
    assert np.isnan(kk[:2]).all() and np.isnan(vv[:2]).all()
    assert np.all(kk[2] == 0)                                 # below the smallest scale
    np.testing.assert_allclose(kk[3], 1e-25, rtol=2.0 ** -21)  # the largest magnitude takes the largest code
    np.testing.assert_allclose(kk[4], 1.0, rtol=2.0 ** -22)
    np.testing.assert_allclose(kk[5, ::2], 3e38, rtol=2.0 ** -21)
    np.testing.assert_array_equal(vv[2:], -kk[2:])


def test_bad_slots_write_nothing_read_nan_and_are_reported():
    cache = PagedKV(2, 64, "e2m1", n_pages=2)
    k = torch.ones(4, 2, 64, device="cuda")
    slots = ints([0, 32, 2 ** 31 - 1, 31])
    cache.append(k, k, slots)
    with pytest.raises(wici.WiciError, match="slot"):
        cache.check()
    codes, each, scales = paged.unpack_e2m1(cache.data.cpu().numpy(), 2, 64)
    for a in (codes, each, scales):
        assert [int(s) for s in np.nonzero(a.reshape(32, -1).any(-1))[0]] == [0, 31]
    got, _ = cache.read(slots, dtype=torch.float32)
    with pytest.raises(wici.WiciError, match="slot"):
        cache.check()
    assert bool(torch.isnan(got[1:3]).all()) and bool(((got[[0, 3]] - 1).abs() < 2.0 ** -20).all())


def test_broadcast_and_odd_aligned_inputs_take_the_narrow_path_to_the_same_bytes():
    rng = np.random.default_rng(3)
    T, kv, d = 40, 2, 64
    k, v = randn(rng, T, kv, d, dtype="bf16"), randn(rng, T, 1, d, dtype="bf16").expand(T, kv, d)
    odd = torch.empty(T * kv * d + 1, dtype=torch.bfloat16, device="cuda")[1:].view(T, kv, d).copy_(k)
    r = Rope(d, 1e4, rot_dim=48)
    datas = []
    for kk, vv in ((k, v), (odd, v), (k, v.contiguous()), (odd, v.contiguous())):
        cache = PagedKV(kv, d, "e2m1", n_pages=3)
        cache.append(kk, vv, ints(range(T)), rope=r, positions=ints(range(T)))
        datas.append(cache.data)
    assert all(torch.equal(datas[0], x) for x in datas[1:])


# ---------------------------------------------------------------- attention --
def attention_case(rng, B, kv, group, d, dtype, lengths, max_pages=None, spread=1.0):
    """A cache whose used slots hold values and whose every other byte is set (codes, NaN scales of both kinds), q, pages."""
    lengths = np.asarray(lengths)
    need = [(max(int(n), 0) + 15) // 16 for n in lengths]
    total = sum(need) + 2
    slots = total * 16
    x = rng.normal(size=(slots, 2, kv, d)) * np.exp(0.5 * rng.normal(size=(2, kv, d)))
    x[:, 1] += 0.2
    codes, each, scales = paged.quantise_e2m1(x.astype(np.float32))
    vals = paged.e2m1_values(codes, each, scales)
    order = rng.permutation(total)
    pages = np.full((len(lengths), max_pages or max(max(need), 1)), -1)
    used = np.zeros(slots, bool)
    at = 0
    for b, n in enumerate(need):
        pages[b, :n] = order[at:at + n]
        t = np.arange(max(int(lengths[b]), 0))
        used[pages[b, t // 16] * 16 + t % 16] = True
        at += n
    codes[~used], each[~used], scales[~used] = 15, 255, np.nan
    data = torch.tensor(paged.pack_e2m1(codes, each, scales), device="cuda")
    q = randn(rng, len(lengths), kv * group, d, dtype=dtype, scale=spread)
    return PagedKV(kv, d, "e2m1", data=data), q, pages, vals


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
    ("bf16", 1, 12, 128, [700, 65, 63, 64], 0),
    ("f32", 1, 33, 64, [140], 0),
])
def test_attention(dtype, kv, group, d, lengths, window):
    rng = np.random.default_rng(len(lengths) * 100 + group)
    cache, q, pages, vals = attention_case(rng, len(lengths), kv, group, d, dtype, lengths)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    for out_dtype in {dtype, "f32"}:
        out = torch.full(q.shape, 7.0, dtype=DT[out_dtype], device="cuda")
        cache.attend(q, ints(pages), ints(lengths), window=window, out=out, lse=lse)
        cache.check()
        check_attention(cache, q, pages, lengths, vals, d ** -0.5, window, out, lse, dtype, out_dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_over_a_long_cache_of_few_sequences(d):
    rng = np.random.default_rng(11)
    lengths = [9001, 5]
    cache, q, pages, vals = attention_case(rng, 2, 1, 2, d, "bf16", lengths, max_pages=700)
    lse = torch.empty(q.shape[:2], device="cuda")
    for window in (0, 8999, 4000, 100):
        out = cache.attend(q, ints(pages), ints(lengths), window=window, lse=lse)
        check_attention(cache, q, pages, lengths, vals, d ** -0.5, window, out, lse, "bf16")


@pytest.mark.parametrize("d", [64, 128])
def test_attention_at_every_window_around_a_units_ends(d):
    rng = np.random.default_rng(31)
    lengths = [130, 64, 33]
    cache, q, pages, vals = attention_case(rng, 3, 1, 3, d, "f32", lengths)
    for window in list(range(1, 70, 3)) + [127, 128, 129, 130, 131]:
        out = cache.attend(q, ints(pages), ints(lengths), window=window)
        check_attention(cache, q, pages, lengths, vals, d ** -0.5, window, out, None, "f32")


@pytest.mark.parametrize("dtype,group,d", [("f32", 4, 64), ("bf16", 3, 128), ("f16", 12, 128)])
def test_scales_of_either_sign_and_none(dtype, group, d):
    # lengths that end inside a unit: keys that are left out, beside a scale of zero and very small ones
    rng = np.random.default_rng(13)
    cache, q, pages, vals = attention_case(rng, 2, 2, group, d, dtype, [100, 37], spread=8.0)
    v_scales = paged.unpack_e2m1(cache.data.cpu().numpy(), 2, d)[2][:, 1].astype(np.float64)
    q64 = f64(q)
    for scale in (1.0, 0.0, -0.5, 1e-30, -1e-44, -0.0):
        lse = torch.empty(q.shape[:2], device="cuda")
        out = cache.attend(q, ints(pages), ints([100, 37]), scale=scale, lse=lse)
        scale = float(np.float32(scale))
        want, want_lse, weight = paged.paged_attention(q64, vals[:, 0], vals[:, 1], pages, [100, 37], scale)
        for b, n in enumerate([100, 37]):
            slots = pages[b][np.arange(n) // 16] * 16 + np.arange(n) % 16
            for h in range(2 * group):
                k, v, s = vals[slots, 0, h // group], vals[slots, 1, h // group], v_scales[slots, h // group]
                x = k @ q64[b, h] * scale
                p = np.exp(x - want_lse[b, h])
                # the terms of check_attention, and what the scores far apart here bring out: a key's weight times its scale
                # of V is held to 2^-32 of the largest such product, and what is lost of it counts v / scale times
                ds = float(np.max(np.abs(k) @ np.abs(q64[b, h])) * abs(scale)) * (2 * d * 2.0 ** -23 + (2.0 ** -16 if dtype == "f32" else 0.0))
                rel = 2 * ds + 2.0 ** -16 + 2.0 ** -21 + n * 2.0 ** -23
                small = 2.0 ** -32 * (p * s).max() * (np.abs(v) / s[:, None]).sum(0)
                within(f64(out[b, h]), want[b, h], rel * weight[b, h] + small * (1 + rel) + half_step(want[b, h], dtype), f"scale {scale}")
                within(float(lse[b, h]), want_lse[b, h], ds + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -23 * abs(want_lse[b, h]), f"lse, scale {scale}")


def test_queries_that_are_not_finite_stay_in_their_rows():
    rng = np.random.default_rng(14)
    cache, q, pages, vals = attention_case(rng, 2, 1, 12, 128, "bf16", [100, 37])
    kept = q.clone()
    q[0, 3, 5], q[1, 9, 0] = float("nan"), float("inf")
    out = cache.attend(q, ints(pages), ints([100, 37]))
    assert bool(torch.isnan(out[0, 3]).all()) and bool(torch.isnan(out[1, 9]).all())
    out[0, 3], out[1, 9] = cache.attend(kept, ints(pages), ints([100, 37]))[[0, 1], [3, 9]]
    check_attention(cache, kept, pages, [100, 37], vals, 128 ** -0.5, 0, out, None, "bf16")


@pytest.mark.parametrize("shift,score", [(20, -70.0), (34, -70.0), (-40, 20.0)])
@pytest.mark.parametrize("dtype,group,n", [("bf16", 4, 300), ("f32", 3, 300), ("bf16", 12, 300)])
def test_one_key_whose_v_is_of_another_size_than_the_others(dtype, group, n, shift, score):
    """Its weight is e^score of the others', its values 2^shift times theirs: what is lost is 2^-22 of a key's part or 2^-32 of the
    largest one's."""
    rng = np.random.default_rng(40)
    d, odd = 64, 137
    cache = PagedKV(1, d, "e2m1", n_pages=n // 16 + 1)
    k, v = torch.zeros(n, 1, d, device="cuda"), randn(rng, n, 1, d)
    k[odd, 0, 0] = score
    v[odd] *= 2.0 ** shift
    cache.append(k, v, ints(range(n)))
    kk, vv = (f64(t)[:, 0] for t in cache.read(ints(range(n)), dtype=torch.float32))
    q = torch.zeros(1, group, d, device="cuda")
    q[..., 0] = 1.0
    out = cache.attend(q.to(DT[dtype]), ints(np.arange(n // 16 + 1)[None]), ints([n]), scale=1.0, out=torch.empty(1, group, d, device="cuda"))
    p = np.exp(kk[:, 0] - kk[:, 0].max())
    p /= p.sum()
    part = p[:, None] * np.abs(vv)
    top = (p * np.abs(vv).max(1)).max()
    # exponent, sums and their join: 2^-16 of each part as in the other tests; of the heaviest key's weight 2^-32 a key
    within(f64(out[0]), np.broadcast_to(p @ vv, (group, d)), 2.0 ** -16 * part.sum(0) + n * 2.0 ** -32 * top + 1e-30, "out")


def test_attention_of_many_ragged_sequences():
    rng = np.random.default_rng(12)
    lengths = rng.integers(0, 120, 300)
    lengths[[5, 299]] = 0
    cache, q, pages, vals = attention_case(rng, 300, 1, 2, 64, "bf16", lengths)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = cache.attend(q, ints(pages), ints(lengths), lse=lse)
    check_attention(cache, q, pages, lengths, vals, 0.125, 0, out, lse, "bf16")
    assert torch.equal(out, cache.attend(q, ints(pages), ints(lengths)))


def test_bad_pages_and_lengths_give_nan_and_are_reported():
    rng = np.random.default_rng(17)
    lengths = [40, 70, 20, 16]
    cache, q, pages, vals = attention_case(rng, 4, 2, 2, 128, "bf16", lengths)
    for bad, n, match in ((pages, [40, 70, pages.shape[1] * 16 + 1, 16], "length"), (None, lengths, "page")):
        if bad is None:
            bad = pages.copy()
            bad[2, 1] = cache.n_pages
        out = cache.attend(q, ints(bad), ints(n))
        with pytest.raises(wici.WiciError, match=match):
            cache.check()
        assert bool(torch.isnan(out[2]).all())
        good = [0, 1, 3]
        check_attention(cache, q[good], pages[good], np.array(lengths)[good], vals, 128 ** -0.5, 0, out[good], None, "bf16")


def test_a_key_of_nan_scale_stays_in_its_sequence():
    cache = PagedKV(1, 64, "e2m1", n_pages=4)
    k = torch.ones(40, 1, 64, device="cuda")
    k[25, 0, 3] = float("nan")
    v = torch.ones(40, 1, 64, device="cuda")
    v[35, 0, 3] = float("inf")                                 # in the third page
    cache.append(k, v, ints(range(40)))
    q = torch.ones(3, 2, 64, device="cuda")
    out = cache.attend(q, ints([[0, -1], [1, -1], [2, -1]]), ints([16, 16, 8]))
    assert bool(((out[0] - 1).abs() < 2.0 ** -20).all()) and bool(torch.isnan(out[1:]).all())


def test_a_decode_loop_of_a_batch_captured_and_replayed():
    """Prompts appended at once, then steps (append + attend) as a captured graph whose inputs change between replays."""
    rng = np.random.default_rng(20)
    B, kv, group, d = 3, 2, 4, 128
    H = kv * group
    prompt, steps = [21, 0, 40], 12
    r = Rope(d, 1e4)
    cache = PagedKV(kv, d, "e2m1", data=torch.full((12 * ops.wici_kv_page_bytes(ops.WICI_KV_E2M1, kv, d),), 255, dtype=torch.uint8, device="cuda"))
    pages = rng.permutation(12).reshape(B, 4)
    lengths = np.array(prompt)
    rows = randn(rng, sum(prompt), H + 2 * kv, d, dtype="bf16")
    pos = np.concatenate([np.arange(n) for n in prompt])
    seq = np.concatenate([np.full(n, b) for b, n in enumerate(prompt)])
    cache.append(rows[:, H:H + kv], rows[:, H + kv:], ints(pages[seq, pos // 16] * 16 + pos % 16), rope=r, positions=ints(pos))
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
        lengths = lengths + live
        d_len.copy_(ints(np.where(live, lengths, 0)))
        graph.replay()
        torch.cuda.synchronize()
        used = np.concatenate([pages[b, t // 16] * 16 + t % 16 for b in range(B) for t in [np.arange(lengths[b])]])
        vals = np.zeros((192, 2, kv, d))
        kk, vv = cache.read(ints(used), dtype=torch.float32)
        vals[used, 0], vals[used, 1] = f64(kk), f64(vv)
        check_attention(cache, q_out, pages, np.where(live, lengths, 0), vals, d ** -0.5, 0, out, None, "bf16")
    cache.check()


def test_pages_of_several_layers_side_by_side():
    """A cache whose page_stride is several pages: one layer's pages among others', which stay as they are."""
    rng = np.random.default_rng(9)
    kv, d, layers, n = 2, 64, 3, 5
    page = ops.wici_kv_page_bytes(ops.WICI_KV_E2M1, kv, d)
    pool = torch.tensor(rng.integers(0, 256, n * layers * page), dtype=torch.uint8, device="cuda")
    before = pool.clone()
    own = PagedKV(kv, d, "e2m1", n_pages=n)
    k, v = randn(rng, 70, kv, d), randn(rng, 70, kv, d)
    own.append(k, v, ints(range(70)))
    c = ops.wici_kv_cache(pool.data_ptr() + page, layers * page, n, kv, d, ops.WICI_KV_E2M1)
    st = torch.cuda.current_stream().cuda_stream
    slots = ints(range(70))
    ops.wici_kv_append(st, c, slots.data_ptr(), 70, ops.heads_of(k, d, k.device, "k"), ops.heads_of(v, d, k.device, "v"))
    view = pool.view(n, layers, page)
    assert torch.equal(view[:, [0, 2]], before.view(n, layers, page)[:, [0, 2]])
    got, want = (paged.unpack_e2m1(x.contiguous().cpu().numpy(), kv, d) for x in (view[:, 1], own.data))
    assert all(np.array_equal(a[:70], b[:70]) for a, b in zip(got, want))
