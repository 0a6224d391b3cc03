"""Selection of pages (include/wici_ops.h): outputs that lie between what it reads, and the search among scores of both signs
that bins of equal width do not tell apart.  Selections are defined by whole numbers and single fp32 roundings: equal."""
import numpy as np
import pytest

from oracle import paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2608_24204_gb300 import KeyBounds, PagedKV, ops, wici  # noqa: E402
from tests.test_gpu_ops import f64, ints  # noqa: E402


def test_outputs_between_heads_and_records_are_as_good_as_any():
    kv, d, n, keep = 2, 64, 40, 5
    record = ops.wici_kv_bounds_bytes(kv, d)
    cache = PagedKV(kv, d, "bf16", n_pages=n)
    apart = torch.zeros(n, 1024, dtype=torch.uint8, device="cuda")            # records 1024 bytes apart, the first `record` theirs
    g = torch.Generator(device="cuda").manual_seed(2)
    apart[:, :kv * 2 * d] = torch.randint(0, 256, (n, kv * 2 * d), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    apart[:, kv * 2 * d:record].view(torch.float32)[:, :kv] = 1.0
    rows = torch.randn(2, 4, 2 * d, generator=g, device="cuda")               # heads of q, and as much between them
    q, kept, codes = rows[..., :d], rows.clone(), apart.clone()
    pages, lengths = ints([np.arange(n), np.arange(n)[::-1]]), ints([16 * n - 3, 16 * n])
    stream = torch.cuda.current_stream().cuda_stream
    bounds = ops.wici_kv_bounds(apart.data_ptr(), 1024)
    shape = ops.wici_select_shape(2, n, keep, 1, 1)

    def select(out, held, blocks):
        ops.wici_kv_select(stream, cache.cache, bounds, shape, pages.data_ptr(), lengths.data_ptr(), ops.heads_of(q, d, q.device, "q"), out,
                           held, blocks, cache.status.data_ptr())

    out, blocks = (torch.empty(2, kv, keep, dtype=torch.int32, device="cuda") for _ in range(2))
    held = torch.empty(2, dtype=torch.int32, device="cuda")
    select(out.data_ptr(), held.data_ptr(), blocks.data_ptr())
    gap, hole = rows[0, 1, d:].data_ptr(), apart[7, record:].data_ptr()       # 256 and 480 bytes that are nobody's
    select(gap, hole, hole + 16)
    assert torch.equal(rows[..., :d], kept[..., :d]) and torch.equal(apart[:, :record], codes[:, :record])
    assert torch.equal(rows[0, 1, d:d + 2 * kv * keep].view(torch.int32), out.flatten())
    assert torch.equal(apart[7, record:record + 8].view(torch.int32), held)
    assert torch.equal(apart[7, record + 16:record + 16 + 8 * kv * keep].view(torch.int32), blocks.flatten())
    for bad in ((gap - 4, hole, hole + 16), (gap + 4 * d - 72, hole, hole + 16), (gap, hole - 8, hole + 16), (gap, hole, apart[8].data_ptr() - 72)):
        with pytest.raises(wici.WiciError, match="overlap"):
            select(*bad)
    cache.check()


def check_search(scales, codes, q, keeps):
    """One sequence of a page for each scale, in any order; q and codes [pages, 2] meet in their first element."""
    n, d = len(scales), q.shape[-1]
    rng = np.random.default_rng(n)
    cache = PagedKV(1, d, "bf16", n_pages=n)
    bounds = KeyBounds(cache)
    bounds.codes[:, 0, :, 0] = torch.tensor(codes, dtype=torch.int8, device="cuda")
    bounds.scales.copy_(torch.tensor(scales, device="cuda")[:, None])
    order = rng.permutation(n)
    scores = paged.page_scores(f64(q)[0], bounds.codes[:, 0].cpu().numpy()[order], scales[order])
    for keep in keeps:
        blocks = torch.empty(1, 1, keep, dtype=torch.int32, device="cuda")
        chosen, held = bounds.select(q, ints(order[None]), ints([16 * n - 5]), keep, first=1, recent=1, blocks=blocks)
        want = paged.selected_pages(scores, keep, 1, 1)
        assert blocks[0, 0].tolist() == want and chosen[0, 0].tolist() == order[want].tolist() and held.tolist() == [16 * keep - 5]
    cache.check()
    return scores


@pytest.mark.parametrize("size", [1e-30, 1.0, 1e30])
def test_negative_scores_beside_infinite_ones(size):
    # pages of NaN scale score +infinity: the scores' width is no number, and their orders differ in the first bit
    rng = np.random.default_rng(5)
    n = 3000
    scales = (rng.uniform(0.5, 2, n) * size).astype(np.float32)
    scales[::7] = np.nan
    q = torch.zeros(1, 1, 64, device="cuda")
    q[..., 0] = -1.0
    scores = check_search(scales, np.full((n, 2), 100), q, (3, 200, 428, 429, 431, 900, 2990))
    assert np.isinf(scores).sum() == 429 and (scores < 0).sum() == n - 429


@pytest.mark.parametrize("top", [1e3, 1e25])
def test_small_scores_of_both_signs_beside_a_large_one(top):
    # all but one score in one bin of equal width, more than are compared one with another
    rng = np.random.default_rng(6)
    n = 2500
    scales = rng.uniform(0.5, 2, n).astype(np.float32) * np.float32(1e-8)
    scales[rng.integers(0, n, 300)] = np.float32(0.75e-8)                      # equal ones among them
    codes = rng.integers(-127, 128, n).repeat(2).reshape(n, 2)
    scales[1234], codes[1234] = top, 127
    q = torch.zeros(1, 2, 64, device="cuda")
    q[0, :, 0] = torch.tensor([1.0, 0.25])
    scores = check_search(scales, codes, q, (2, 3, 4, 600, 1249, 1251, 1400, 2400))
    assert (scores > 0).sum() > 1000 and (scores < 0).sum() > 1000


@pytest.mark.parametrize("batch,kv,most", [(32, 8, 3000), (40, 8, 2049), (20, 8, 8192), (160, 1, 6000)])
def test_more_sequences_and_heads_than_sms_over_many_pages(batch, kv, most):
    """Blocks of either size, in several waves: short sequences beside long ones, some with nothing to choose."""
    d, group, keep, total = 128, 4, 60, 16384
    g = torch.Generator(device="cuda").manual_seed(most)
    cache = PagedKV(kv, d, "e2m1", n_pages=total)
    bounds = KeyBounds(cache)
    bounds.codes.copy_(torch.randint(-127, 128, bounds.codes.shape, generator=g, device="cuda", dtype=torch.int32))
    bounds.scales.copy_(torch.rand(bounds.scales.shape, generator=g, device="cuda") + 0.5)
    q = torch.randn((batch, kv * group, d), generator=g, device="cuda").bfloat16()
    pages = torch.randint(0, total, (batch, most), generator=g, device="cuda", dtype=torch.int32)   # sequences may share pages
    lengths = torch.randint(1, 16 * most + 1, (batch,), generator=g, device="cuda", dtype=torch.int32)
    lengths[:6] = ints([0, 1, 16 * keep, 16 * keep + 1, 16 * most, 16 * most - 15])
    blocks = torch.empty(batch, kv, keep, dtype=torch.int32, device="cuda")
    chosen, held = bounds.select(q, pages, lengths, keep, first=1, recent=3, blocks=blocks)
    cache.check()
    m = q.float().abs().amax(-1, keepdim=True)
    w = (q.float() * (m.reciprocal() * 1023.0)).round().double().view(batch, kv, group, d)
    for b, n in enumerate(lengths.tolist()):
        count = -(-n // 16)
        at = pages[b, :count].long()
        c = bounds.codes[at].double()                                          # [pages, kv, 2, d]
        dot = torch.einsum("hgd,phd->hgp", w[b].clamp_min(0), c[:, :, 0]) + torch.einsum("hgd,phd->hgp", w[b].clamp_max(0), c[:, :, 1])
        score = ((dot.float() * m[b].view(kv, group, 1)).amax(1) * bounds.scales[at].T).cpu().numpy()
        for h in range(kv):
            want = paged.selected_pages(score[h], keep, 1, 3) if count else []
            assert blocks[b, h].tolist() == want + [-1] * (keep - len(want))
            assert chosen[b, h, :len(want)].tolist() == at[want].tolist()
        assert held[b].item() == (n if count <= keep else (keep - 1) * 16 + (n - 1) % 16 + 1)
