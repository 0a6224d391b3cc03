"""Bounds of a cache's pages, the selection of pages by them, and attention where every KV head has pages of its own
(include/wici_ops.h) through their binding, against the oracle (oracle/paged.py).

Bounds and scores are defined by whole numbers and single fp32 roundings: codes, scales and selections have to be equal.
Attention's tolerances are those of tests/test_gpu_ops.py.
"""
import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import gen  # noqa: E402
from paper_2608_24204_gb300 import KeyBounds, PagedKV, Rope, WiciModel, ops, wici  # noqa: E402
from tests.test_gpu_ops import DT, check_attention, f64, ints, randn  # noqa: E402


def filled(rng, pages, kv, d, fmt, spread=1.0):
    """A cache whose every slot holds a token, and its values [slots, 2, kv, d] as fp32 has them."""
    cache = PagedKV(kv, d, fmt, n_pages=pages)
    topic = rng.normal(size=(pages, 1, kv, d)).repeat(16, 1).reshape(pages * 16, kv, d)
    k = torch.tensor((rng.normal(size=(pages * 16, kv, d)) + topic) * spread, device="cuda").float()
    cache.append(k, randn(rng, pages * 16, kv, d), ints(range(pages * 16)))
    vals = np.stack([f64(t) for t in cache.read(ints(range(pages * 16)), dtype=torch.float32)], 1)
    return cache, vals


def want_bounds(vals, page, rows):
    kv = vals.shape[2]
    got = [paged.key_bounds(vals[page * 16:page * 16 + rows, 0, h]) for h in range(kv)]
    return np.stack([c for c, _ in got]), np.array([s for _, s in got])


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3", "e2m1"])
@pytest.mark.parametrize("kv,d,pages", [(1, 64, 3), (8, 128, 20), (3, 64, 40), (5, 128, 7)])
def test_bounds(fmt, kv, d, pages):
    rng = np.random.default_rng(pages)
    cache, vals = filled(rng, pages, kv, d, fmt)
    data = torch.full((pages * ops.wici_kv_bounds_bytes(kv, d),), 99, dtype=torch.uint8, device="cuda")
    bounds = KeyBounds(cache, data=data)
    before = bounds.codes.clone(), bounds.scales.clone(), data.clone()
    some = rng.permutation(pages)[:max(1, pages * 2 // 3)]
    rows = rng.integers(1, 17, len(some))
    rows[0] = 16
    last = some * 16 + rows - 1
    bounds.update(ints(np.concatenate([last, [-1, -2 ** 31]])))
    cache.check()
    codes, scales = bounds.codes.cpu().numpy(), bounds.scales.cpu().numpy()
    for p, r in zip(some, rows):
        c, s = want_bounds(vals, p, r)
        np.testing.assert_array_equal(scales[p], s)
        np.testing.assert_array_equal(codes[p], c)
    others = torch.tensor(sorted(set(range(pages)) - set(some.tolist())), dtype=torch.long, device="cuda")
    assert torch.equal(bounds.codes[others], before[0][others]) and torch.equal(bounds.scales[others].view(torch.int32), before[1][others].view(torch.int32))
    record = ops.wici_kv_bounds_bytes(kv, d)
    assert torch.equal(data.view(pages, record)[:, kv * (2 * d + 4):], before[2].view(pages, record)[:, kv * (2 * d + 4):])


def test_bounds_of_infinite_zero_and_tiny_keys_and_of_slots_outside():
    cache = PagedKV(1, 64, "bf16", n_pages=5)
    k = torch.ones(80, 1, 64, device="cuda")
    k[3, 0, 5], k[20, 0, 63], k[32:48], k[48:64] = float("inf"), float("nan"), 0, 2.0 ** -125
    k[66, 0, 1] = -3.0
    cache.append(k, k, ints(range(80)))
    bounds = KeyBounds(cache)
    bounds.update(ints([2, 15 + 16, 47, 63, 79]))
    assert bounds.scales.flatten().isnan().tolist() == [False, True, False, False, False]
    assert bounds.scales[2:4].flatten().tolist() == [0, 0] and not bool(bounds.codes[1:4].any())
    assert bounds.scales[0].item() == float(np.float32(1) / np.float32(127)) and bool((bounds.codes[0] == 127).all())
    assert bounds.codes[4, 0, 1, 1].item() == -127 and bounds.codes[4, 0, 0, 1].item() == 42
    bounds.update(ints([3]))
    assert bool(bounds.scales[0].isnan().all())               # the place of the infinity is in the page's part now
    kept = bounds.data.clone()
    cache.check()
    bounds.update(ints([80, 2 ** 31 - 1, -5]))
    with pytest.raises(wici.WiciError, match="slot"):
        cache.check()
    assert torch.equal(kept, bounds.data)
    bounds.update(ints([]))


def selection_case(rng, kv, group, d, fmt, dtype, lengths, max_pages=None, spread=1.0):
    lengths = np.asarray(lengths)
    need = [(max(int(n), 0) + 15) // 16 for n in lengths]
    total = sum(need) + 2
    cache, vals = filled(rng, total, kv, d, fmt, spread)
    order = rng.permutation(total)
    pages = np.full((len(lengths), max_pages or max(max(need), 1)), -1)
    at, last = 0, []
    for b, n in enumerate(need):
        pages[b, :n] = order[at:at + n]
        at += n
        last += [p * 16 + 15 for p in pages[b, :n - 1]] + ([pages[b, n - 1] * 16 + (lengths[b] - 1) % 16] if n else [])
    bounds = KeyBounds(cache)
    bounds.update(ints(last))
    return cache, bounds, randn(rng, len(lengths), kv * group, d, dtype=dtype), pages, vals


def want_selection(bounds, q, pages, lengths, keep, first, recent):
    codes, scales = bounds.codes.cpu().numpy(), bounds.scales.cpu().numpy()
    B, kv = len(lengths), codes.shape[1]
    q = q.float().cpu().numpy().reshape(B, kv, -1, q.shape[2])
    blocks = np.full((B, kv, keep), -1)
    held = np.zeros(B, int)
    for b, n in enumerate(lengths):
        count = (max(int(n), 0) + 15) // 16
        for h in range(kv):
            p = pages[b, :count]
            s = paged.page_scores(q[b, h], codes[p, h], scales[p, h]) if count > keep else np.zeros(count)
            chosen = paged.selected_pages(s, keep, first, recent)
            blocks[b, h, :len(chosen)] = chosen
        held[b] = max(int(n), 0) if count <= keep else (keep - 1) * 16 + (int(n) - 1) % 16 + 1
    chosen = np.where(blocks >= 0, np.take_along_axis(np.repeat(pages[:, None], kv, 1), np.maximum(blocks, 0), -1), -1)
    return chosen, held, blocks


def check_selected(cache, bounds, q, pages, lengths, vals, keep, first, recent, dtype):
    """Selection and the attention over it; a KV head's attention is that of a cache with its pages."""
    B, kv = len(lengths), cache.n_kv_heads
    blocks = torch.full((B, kv, keep), 7, dtype=torch.int32, device="cuda")
    chosen, held = bounds.select(q, ints(pages), ints(lengths), keep, first=first, recent=recent, blocks=blocks)
    want = want_selection(bounds, q, pages, lengths, keep, first, recent)
    np.testing.assert_array_equal(held.cpu().numpy(), want[1])
    np.testing.assert_array_equal(blocks.cpu().numpy(), want[2])
    np.testing.assert_array_equal(chosen.cpu().numpy(), want[0])
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = cache.attend(q, chosen, held, lse=lse)
    cache.check()
    group = q.shape[1] // kv
    for h in range(kv):
        part = slice(h * group, (h + 1) * group)
        check_attention(cache, q[:, part].contiguous(), want[0][:, h], want[1], vals[:, :, h:h + 1], q.shape[2] ** -0.5, 0, out[:, part], lse[:, part], dtype)
    return chosen, held, out


@pytest.mark.parametrize("dtype,fmt,kv,group,d,lengths,keep,first,recent", [
    ("bf16", "bf16", 1, 1, 128, [1], 1, 0, 1),
    ("f32", "int8", 2, 4, 64, [0, 1, 16, 17, 33, 100, 160], 3, 1, 1),
    ("bf16", "e2m1", 8, 4, 128, [300, 0, 129, 1, 700], 5, 1, 2),
    ("f16", "e4m3", 3, 5, 128, [270, 257, 16], 4, 0, 1),
    ("bf16", "bf16", 2, 9, 64, [900, 331], 20, 4, 8),
    ("f32", "bf16", 1, 16, 128, [555, 1000], 7, 0, 7),        # nothing is scored for
    ("bf16", "e2m1", 1, 64, 64, [500], 2, 1, 1),
    ("f16", "int8", 4, 7, 64, [513, 512, 511, 528], 32, 1, 1),
    ("bf16", "bf16", 2, 2, 64, [4113], 33, 2, 3),
    ("f32", "e2m1", 1, 3, 128, [2000, -5], 124, 0, 4),
])
def test_selection_and_attention_over_it(dtype, fmt, kv, group, d, lengths, keep, first, recent):
    rng = np.random.default_rng(sum(lengths) + keep)
    cache, bounds, q, pages, vals = selection_case(rng, kv, group, d, fmt, dtype, lengths)
    check_selected(cache, bounds, q, pages, lengths, vals, keep, first, recent, dtype)


@pytest.mark.parametrize("n,keep,batch,kv,d", [(20000, 40, 1, 1, 64), (9000, 100, 3, 2, 128), (3000, 8, 40, 1, 64), (2000, 16, 24, 8, 64),
                                                (6000, 30, 20, 8, 128), (9000, 50, 50, 8, 64), (100000, 900, 2, 1, 64)])
def test_long_contexts_and_many_sequences(n, keep, batch, kv, d):
    # every number of blocks that share a sequence
    rng = np.random.default_rng(n)
    lengths = [n] + rng.integers(0, n, batch - 1).tolist()
    total = sum((x + 15) // 16 for x in lengths)
    bounds_of = KeyBounds(PagedKV(kv, d, "bf16", n_pages=total + 1))
    g = torch.Generator(device="cuda").manual_seed(n)
    bounds_of.codes.copy_(torch.randint(-127, 128, bounds_of.codes.shape, generator=g, device="cuda", dtype=torch.int32))
    bounds_of.scales.copy_(torch.rand(bounds_of.scales.shape, generator=g, device="cuda") + 0.5)
    pages = np.full((batch, n // 16 + 3), -1)
    order, at = rng.permutation(total + 1), 0
    for b, x in enumerate(lengths):
        c = (x + 15) // 16
        pages[b, :c] = order[at:at + c]
        at += c
    q = randn(rng, batch, kv * 2, d, dtype="bf16")
    blocks = torch.empty((batch, kv, keep), dtype=torch.int32, device="cuda")
    chosen, held = bounds_of.select(q, ints(pages), ints(lengths), keep, first=1, recent=2, blocks=blocks)
    # the oracle's scores with the products of whole numbers as one matrix product in 64 bits
    x = q.float().view(batch, kv, 2, d)
    m = x.abs().amax(-1, keepdim=True)
    w = (x * (m.reciprocal() * 1023.0)).round().double()
    c = bounds_of.codes.double()
    for b, length in enumerate(lengths):
        count = (length + 15) // 16
        p = torch.tensor(pages[b, :count], device="cuda").long()
        dots = torch.einsum("hgd,phd->hgp", w[b].clamp_min(0), c[p, :, 0]) + torch.einsum("hgd,phd->hgp", w[b].clamp_max(0), c[p, :, 1])
        score = (dots.float() * m[b]).amax(1) * bounds_of.scales[p].T
        for h in range(kv):
            want = paged.selected_pages(score[h].cpu().numpy(), keep, 1, 2)
            assert blocks[b, h].tolist() == want + [-1] * (keep - len(want))
            assert chosen[b, h].tolist() == [pages[b, i] for i in want] + [-1] * (keep - len(want))
    again = bounds_of.select(q, ints(pages), ints(lengths), keep, first=1, recent=2)
    assert torch.equal(again[0], chosen) and torch.equal(again[1], held)


def test_equal_scores_go_to_the_first_pages():
    cache = PagedKV(2, 64, "bf16", n_pages=100)
    bounds = KeyBounds(cache)
    bounds.codes.fill_(1)
    bounds.scales.fill_(1.0)
    bounds.scales[70:80, 0] = 2.0
    bounds.codes[50:60, 1] = -1
    q = torch.ones(1, 2, 64, device="cuda")
    pages = ints(np.arange(100)[None])
    blocks = torch.empty(1, 2, 20, dtype=torch.int32, device="cuda")
    bounds.select(q, pages, ints([1600]), 20, first=2, recent=1, blocks=blocks)
    assert blocks[0, 0].tolist() == list(range(2)) + list(range(2, 9)) + list(range(70, 80)) + [99]
    assert blocks[0, 1].tolist() == list(range(19)) + [99]
    bounds.select(-q, pages, ints([1600]), 20, first=0, recent=1, blocks=blocks)
    assert blocks[0, 0].tolist() == list(range(19)) + [99]    # the ten of larger scale are the lowest
    assert blocks[0, 1].tolist() == list(range(9)) + list(range(50, 60)) + [99]
    bounds.scales.zero_()
    bounds.select(q, pages, ints([1600]), 20, first=0, recent=4, blocks=blocks)
    assert blocks[0, 0].tolist() == list(range(16)) + [96, 97, 98, 99]


@pytest.mark.parametrize("kinds", [1, 2, 5])
@pytest.mark.parametrize("huge", [False, True])
def test_many_equal_scores_of_a_few_kinds(kinds, huge):
    # more of them than are compared one by one, in one bin; scores whose differences fp32 does not hold
    rng = np.random.default_rng(kinds)
    n, d = 3000, 64
    cache = PagedKV(1, d, "bf16", n_pages=n)
    bounds = KeyBounds(cache)
    bounds.codes.fill_(100)
    size = (np.array([1.0, 1.0 + 2.0 ** -23, 1.0 + 2.0 ** -22, 0.999, 3.0]) * (1e30 if huge else 1.0)).astype(np.float32)
    scales = size[rng.integers(0, kinds, n)]
    if huge:
        scales[::7] = np.nan
    bounds.scales.copy_(torch.tensor(scales, device="cuda")[:, None])
    q = torch.full((1, 1, d), 1e10, device="cuda") * torch.where(torch.arange(d, device="cuda") % 2 == 0, 1.0, -1.0)
    q[..., :2] = 1e10
    pages = ints(rng.permutation(n)[None])
    for keep in (3, 500, 1400, 2999):
        blocks = torch.empty(1, 1, keep, dtype=torch.int32, device="cuda")
        chosen, held = bounds.select(q, pages, ints([16 * n - 5]), keep, first=1, recent=1, blocks=blocks)
        scores = paged.page_scores(f64(q)[0], bounds.codes[:1, 0].cpu().numpy().repeat(n, 0), scales[pages[0].cpu().numpy()])
        want = paged.selected_pages(scores, keep, 1, 1)
        assert blocks[0, 0].tolist() == want
        assert chosen[0, 0].tolist() == pages[0, want].tolist() and held.tolist() == [16 * keep - 5]


def test_the_largest_call():
    """The most pages, pages to select and query heads of a KV head."""
    n, keep, d, group = 16384, 4096, 128, 64
    cache = PagedKV(1, d, "e2m1", n_pages=n)
    bounds = KeyBounds(cache)
    g = torch.Generator(device="cuda").manual_seed(1)
    bounds.codes.copy_(torch.randint(-127, 128, bounds.codes.shape, generator=g, device="cuda", dtype=torch.int32))
    bounds.scales.copy_(torch.rand(bounds.scales.shape, generator=g, device="cuda") + 0.5)
    q = torch.randn((1, group, d), generator=g, device="cuda")
    pages = torch.randperm(n, generator=g, device="cuda").int()[None]
    blocks = torch.empty(1, 1, keep, dtype=torch.int32, device="cuda")
    chosen, held = bounds.select(q, pages, ints([16 * n]), keep, first=3, recent=5, blocks=blocks)
    m = q.abs().amax(-1, keepdim=True)
    w = (q * (m.reciprocal() * 1023.0)).round().double()[0]
    c = bounds.codes[pages[0].long(), 0].double()
    score = ((w.clamp_min(0) @ c[:, 0].T + w.clamp_max(0) @ c[:, 1].T).float() * m[0]).amax(0) * bounds.scales[pages[0].long(), 0]
    want = paged.selected_pages(score.cpu().numpy(), keep, 3, 5)
    assert blocks[0, 0].tolist() == want and held.tolist() == [16 * keep]
    assert torch.equal(chosen[0, 0], pages[0, torch.tensor(want, device="cuda")])


def test_first_calls_of_a_process_inside_a_capture():
    """Set-up that a first call makes must not need a call before the capture (attention's is made with the cache)."""
    code = """
import torch
from paper_2608_24204_gb300 import KeyBounds, PagedKV
cache = PagedKV(2, 64, "e2m1", n_pages=200)
bounds = KeyBounds(cache)
q = torch.randn(1, 4, 64, device="cuda")
pages, n = torch.arange(200, device="cuda", dtype=torch.int32)[None], torch.tensor([3200], device="cuda", dtype=torch.int32)
k = torch.randn(3200, 2, 64, device="cuda")
slots = torch.arange(3200, device="cuda", dtype=torch.int32)
last = torch.arange(15, 3200, 16, device="cuda", dtype=torch.int32)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    cache.append(k, k, slots)
    bounds.update(last)
    chosen, held = bounds.select(q, pages, n, 20)
    out = cache.attend(q, chosen, held)
graph.replay()
torch.cuda.synchronize()
cache.check()
chosen2, held2 = bounds.select(q, pages, n, 20)
assert torch.equal(chosen, chosen2) and held2.item() == 320 and torch.equal(out, cache.attend(q, chosen2, held2))
print("fine")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout + r.stderr


def test_largest_products_stay_exact():
    """Every product at its largest, and pages that differ by one unit of one code."""
    d, n = 128, 64
    cache = PagedKV(1, d, "bf16", n_pages=n)
    bounds = KeyBounds(cache)
    bounds.codes[:, :, 0], bounds.codes[:, :, 1] = 127, -127
    rng = np.random.default_rng(5)
    less = rng.permutation(n)
    for p in range(n):                                         # page p lacks less[p] units of one
        left = int(less[p])
        for e in range(d):
            cut = min(left, 1)
            bounds.codes[p, 0, 0, e] -= cut
            bounds.codes[p, 0, 1, e] += cut
            left -= cut
    bounds.scales.fill_(1.0)
    sign = torch.tensor(rng.choice([-1.0, 1.0], d), device="cuda")
    blocks = torch.empty(1, 1, 21, dtype=torch.int32, device="cuda")
    for size in (1.0, 2.0 ** -90, 1.5 * 2.0 ** 100):
        bounds.select((sign * size).float().view(1, 1, d), ints(np.arange(n)[None]), ints([16 * n]), 21, first=0, recent=1, blocks=blocks)
        rest = sorted(range(n - 1), key=lambda p: less[p])[:20]
        assert blocks[0, 0].tolist() == sorted(rest) + [n - 1]


def test_bounds_contain_their_keys_and_rank_by_the_largest_product():
    """The score is at least every q.k of its page, to the roundings of codes and of q."""
    rng = np.random.default_rng(6)
    cache, vals = filled(rng, 30, 1, 64, "bf16")
    bounds = KeyBounds(cache)
    bounds.update(ints(np.arange(30) * 16 + 15))
    q = rng.normal(size=(1, 64)).astype(np.float32)
    s = paged.page_scores(q, bounds.codes.cpu().numpy()[:, 0], bounds.scales.cpu().numpy()[:, 0]) / 1023
    most = (vals[:, 0, 0].reshape(30, 16, 64) @ q[0].astype(np.float64)).max(1)
    slack = np.abs(q).sum() * bounds.scales.cpu().numpy()[:, 0] * 0.5 + np.abs(q).max() / 1023 * 0.5 * np.abs(vals[:, 0, 0]).reshape(30, 16, 64).max(1).sum(-1)
    assert np.all(s >= most - slack * 1.01)


def test_queries_and_pages_that_are_not_finite():
    rng = np.random.default_rng(7)
    cache, bounds, q, pages, vals = selection_case(rng, 2, 2, 64, "bf16", "f32", [640, 640, 640])
    q[0, 1, 3], q[1, 2:, 0], q[1, 2:, 1:] = float("nan"), 1e-38, 0
    q[1, 0, 7] = float("inf")
    bounds.scales[int(pages[2, 11]), 0] = float("nan")
    bounds.scales[int(pages[2, 17]), 1] = float("inf")
    blocks = torch.empty(3, 2, 6, dtype=torch.int32, device="cuda")
    bounds.select(q, ints(pages), ints([640] * 3), 6, first=0, recent=1, blocks=blocks)
    want = want_selection(bounds, q, pages, [640] * 3, 6, 0, 1)
    np.testing.assert_array_equal(blocks.cpu().numpy(), want[2])
    assert 11 in blocks[2, 0].tolist() and 17 in blocks[2, 1].tolist()
    assert blocks[1, 1].tolist() == [0, 1, 2, 3, 4, 39]       # queries of no size: the first pages


def test_bad_pages_and_lengths_are_reported_and_stay_bad():
    rng = np.random.default_rng(8)
    cache, bounds, q, pages, vals = selection_case(rng, 1, 2, 64, "int8", "bf16", [300, 300, 40])
    for long in (True, False):
        bad, n = pages.copy(), [300, 300, 40]
        if long:
            n[1] = pages.shape[1] * 16 + 1
        else:
            bad[1, 5] = cache.n_pages                          # scores first
            bad[2, 1] = -3                                     # all of this one's pages are taken
        chosen, held = bounds.select(q, ints(bad), ints(n), 4)
        with pytest.raises(wici.WiciError, match="length" if long else "page"):
            cache.check()
        out = cache.attend(q, chosen, held)
        with pytest.raises(wici.WiciError, match="length" if long else "page"):
            cache.check()
        assert bool(torch.isnan(out[1]).all()) and bool(torch.isfinite(out[0]).all())
        assert bool(torch.isnan(out[2]).all()) is not long


def test_rows_of_strided_queries_and_other_heads_pages():
    rng = np.random.default_rng(9)
    cache, bounds, _, pages, vals = selection_case(rng, 2, 3, 64, "e2m1", "bf16", [500, 64, 210])
    big = randn(rng, 6, 5, 65, dtype="bf16")
    q = big.transpose(0, 1)[:3, :, 1:]                         # heads first, 2-byte aligned
    check_selected(cache, bounds, q, pages, [500, 64, 210], vals, 6, 1, 2, "bf16")


def test_attention_of_selected_pages_matches_the_ordinary_one_where_all_are_selected():
    rng = np.random.default_rng(10)
    for fmt, dtype, group in (("bf16", "bf16", 4), ("e2m1", "f32", 9), ("int8", "f16", 16)):
        lengths = [333, 16, 0, 1]
        cache, bounds, q, pages, vals = selection_case(rng, 2, group, 128, fmt, dtype, lengths)
        chosen, held = bounds.select(q, ints(pages), ints(lengths), pages.shape[1])
        assert held.tolist() == lengths
        assert torch.equal(cache.attend(q, chosen, held), cache.attend(q, ints(pages), ints(lengths)))
    with pytest.raises(wici.WiciError, match="window"):
        cache.attend(q, chosen, held, window=3)


def test_a_context_grows_under_a_captured_step():
    """append, update, select and attend of a batch as one captured graph: every step against the oracle on what the
    cache and its bounds then hold."""
    rng = np.random.default_rng(20)
    B, kv, group, d, columns, keep = 3, 2, 4, 64, 8, 3
    H = kv * group
    prompt, steps = [90, 0, 40], 20
    r = Rope(d, 1e4)
    cache = PagedKV(kv, d, "e2m1", n_pages=B * columns)
    bounds = KeyBounds(cache)
    pages = rng.permutation(B * columns).reshape(B, columns)
    lengths = np.array(prompt)
    rows = randn(rng, sum(prompt), H + 2 * kv, d, dtype="bf16")
    pos = np.concatenate([np.arange(n) for n in prompt])
    seq = np.concatenate([np.full(n, b) for b, n in enumerate(prompt)])
    slots = pages[seq, pos // 16] * 16 + pos % 16
    cache.append(rows[:, H:H + kv], rows[:, H + kv:], ints(slots), rope=r, positions=ints(pos))
    ends = (pos % 16 == 15) | (pos == np.array(prompt)[seq] - 1)
    bounds.update(ints(slots[ends]))
    step = torch.zeros(B, H + 2 * kv, d, dtype=torch.bfloat16, device="cuda")
    q_out, out = torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda")
    d_pos, d_slots, d_len, d_pages = ints([0] * B), ints([-1] * B), ints([0] * B), ints(pages)
    sel = torch.empty(B, kv, keep, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    blocks = torch.empty(B, kv, keep, dtype=torch.int32, device="cuda")

    def one():
        cache.append(step[:, H:H + kv], step[:, H + kv:], d_slots, rope=r, positions=d_pos, q=step[:, :H], q_out=q_out)
        bounds.update(d_slots)
        bounds.select(q_out, d_pages, d_len, keep, first=1, recent=1, out=sel, blocks=blocks)
        cache.attend(q_out, *sel, out=out)

    one()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for s in range(steps):
        live = np.array([True, True, s % 3 != 0])
        step.copy_(randn(rng, B, H + 2 * kv, d, dtype="bf16"))
        slot = np.where(live, pages[np.arange(B), lengths // 16] * 16 + lengths % 16, -1)
        d_pos.copy_(ints(lengths))
        d_slots.copy_(ints(slot))
        lengths = lengths + live
        now = np.where(live, lengths, 0)
        d_len.copy_(ints(now))
        graph.replay()
        torch.cuda.synchronize()
        used = np.concatenate([pages[b, t // 16] * 16 + t % 16 for b in range(B) for t in [np.arange(lengths[b])]])
        vals = np.zeros((B * columns * 16, 2, kv, d))
        kk, vv = cache.read(ints(used), dtype=torch.float32)
        vals[used, 0], vals[used, 1] = f64(kk), f64(vv)
        for b in range(B):
            for i in range((lengths[b] + 15) // 16):
                c, sc = want_bounds(vals, int(pages[b, i]), min(16, lengths[b] - 16 * i))
                assert np.array_equal(bounds.codes[int(pages[b, i])].cpu().numpy(), c)
                assert np.array_equal(bounds.scales[int(pages[b, i])].cpu().numpy(), sc)
        want = want_selection(bounds, q_out, pages, now, keep, 1, 1)
        np.testing.assert_array_equal(sel[0].cpu().numpy(), want[0])
        np.testing.assert_array_equal(sel[1].cpu().numpy(), want[1])
        np.testing.assert_array_equal(blocks.cpu().numpy(), want[2])
        for h in range(kv):
            part = slice(h * group, (h + 1) * group)
            check_attention(cache, q_out[:, part].contiguous(), want[0][:, h], want[1], vals[:, :, h:h + 1], d ** -0.5, 0, out[:, part], None, "bf16")
    cache.check()


def test_a_contexts_prompt_attended_in_part():
    """A model's own cache (wici_kv_view) under bounds: select and attend on its pages."""
    cfg = gen.TINY
    model = WiciModel(cfg, max_tokens=96).load(gen.make_weights(cfg))
    model.prefill(gen.make_prompt(cfg, 70, seed=1))
    torch.cuda.synchronize()
    cache, table = model.kv_cache(1)
    n = 70
    pages = table[:(n + 15) // 16].view(1, -1).contiguous()
    bounds = KeyBounds(cache)
    last = pages[0] * 16 + torch.tensor([15, 15, 15, 15, 5], device="cuda", dtype=torch.int32)
    bounds.update(last)
    q = randn(np.random.default_rng(3), 1, cfg.n_q_heads, cfg.head_dim, dtype="f32")
    kk, vv = model.read_kv(1, dtype=torch.float32)
    vals = np.zeros((cache.n_pages * 16, 2, cfg.n_kv_heads, cfg.head_dim))
    where = (pages[0].cpu().numpy()[:, None] * 16 + np.arange(16)).reshape(-1)[:n]
    vals[where, 0], vals[where, 1] = f64(kk), f64(vv)
    check_selected(cache, bounds, q, pages.cpu().numpy(), [n], vals, 3, 1, 1, "f32")
    model.close()


@pytest.mark.parametrize("fmt,group,batch,kv", [("e2m1", 1, 1100, 2), ("bf16", 3, 1030, 1), ("e2m1", 12, 300, 1), ("int8", 9, 270, 2)])
def test_batches_of_more_sequences_than_a_launch_takes(fmt, group, batch, kv):
    rng = np.random.default_rng(batch)
    lengths = rng.integers(0, 90, batch)
    lengths[-1] = 85
    cache, bounds, q, pages, vals = selection_case(rng, kv, group, 64, fmt, "bf16", lengths)
    chosen, held, out = check_selected(cache, bounds, q, pages, lengths, vals, 3, 1, 1, "bf16")
    lse = torch.empty(q.shape[:2], device="cuda")
    check_attention(cache, q, pages, lengths, vals, 0.125, 0, cache.attend(q, ints(pages), ints(lengths), lse=lse), lse, "bf16")


@pytest.mark.parametrize("fmt,n_pages", [("e2m1", 3_600_000), ("bf16", 1_200_000)])
def test_a_cache_of_more_than_4_gb(fmt, n_pages):
    """Tokens in the last pages, and the same tokens in the first ones of a small cache: the same bounds, lists and results."""
    rng = np.random.default_rng(4)
    n, d = 600, 64
    k, v = randn(rng, n, 1, d), randn(rng, n, 1, d)
    q = randn(rng, 1, 5, d)
    results = []
    for pages_of, first in ((n_pages, n_pages - 38), (38, 0)):
        cache = PagedKV(1, d, fmt, n_pages=pages_of)
        assert pages_of == 38 or cache.data.numel() > 1 << 32
        bounds = KeyBounds(cache)
        slots = first * 16 + np.arange(n)
        cache.append(k, v, ints(slots))
        bounds.update(ints(np.append(slots[15::16], slots[-1])))
        pages = ints((first + np.arange(38))[None])
        blocks = torch.empty(1, 1, 9, dtype=torch.int32, device="cuda")
        chosen, held = bounds.select(q, pages, ints([n]), 9, blocks=blocks)
        assert torch.equal(chosen, blocks + first)
        results.append([bounds.data.view(pages_of, -1)[first:first + 38].clone(), blocks, held, cache.attend(q, chosen, held), cache.attend(q, pages, ints([n])),
                        *cache.read(ints(slots), dtype=torch.float32)])
        cache.check()
        del cache, bounds
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_two_streams_at_once():
    rng = np.random.default_rng(30)
    cases = [selection_case(rng, 2, 4, 128, fmt, "bf16", [1500, 200, 900]) for fmt in ("bf16", "e2m1")]
    tables = [(ints(c[3]), ints([1500, 200, 900])) for c in cases]
    want = [c[0].attend(c[2], *c[1].select(c[2], *t, 12)) for c, t in zip(cases, tables)]
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, (c, t) in enumerate(zip(cases, tables)):
            with torch.cuda.stream(streams[i]):
                got[i].append(c[0].attend(c[2], *c[1].select(c[2], *t, 12)))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for xs, w in zip(got, want) for x in xs)
