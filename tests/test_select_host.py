"""Host-side checks of the bounds, selection and selected attention of include/wici_ops.h: sizes and refusals (arguments
are checked before a device is touched), and pins of their oracle.  No GPU."""
import numpy as np
import pytest

from oracle import paged
from paper_2608_24204_gb300 import build, ops, wici
from tests.test_ops_host import A, cache, heads, refused


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def bounds(kv=8, d=128, data=A, stride=None):
    return ops.wici_kv_bounds(data, ops.wici_kv_bounds_bytes(kv, d) if stride is None else stride)


def test_bounds_bytes():
    assert ops.wici_kv_bounds_bytes(8, 128) == 8 * (2 * 128 + 4)
    assert ops.wici_kv_bounds_bytes(1, 64) == 144 and ops.wici_kv_bounds_bytes(3, 64) == 400
    assert ops.wici_kv_bounds_bytes(8, 96) == ops.wici_kv_bounds_bytes(0, 64) == ops.wici_kv_bounds_bytes(-1, 128) == 0


FAR = [A + (i << 24) for i in range(8)]          # apart from one another


def select(shape=(2, 4, 2, 1, 1), c=None, b=None, pages=FAR[0], lengths=FAR[1], q=None, out=FAR[2], held=FAR[3], blocks=FAR[4],
           status=None, match=""):
    refused(ops.wici_kv_select, 0, c or cache(), b or bounds(), ops.wici_select_shape(*shape), pages, lengths, q or heads(n=32), out,
            held, blocks, status, match=match)


@pytest.mark.parametrize("bad,match", [
    (bounds(data=None), "null"), (bounds(data=A + 8), "aligned"), (bounds(stride=8 * 260 - 16), "page_stride"),
    (bounds(stride=8 * 260 + 8), "page_stride"), (bounds(stride=1 << 62), "page_stride")])
def test_bad_bounds_are_refused(bad, match):
    select(b=bad, match=match)
    refused(ops.wici_kv_bounds_update, 0, cache(), bad, A, 1, match=match)


def test_bad_caches_are_refused():
    for bad, match in ((cache(data=None), "null"), (cache(pages=0), "n_pages"), (ops.wici_kv_cache(A, 1 << 20, 4, 8, 64, 3), "format")):
        select(c=bad, match=match)
        refused(ops.wici_kv_bounds_update, 0, bad, bounds(), A, 1, match=match)


@pytest.mark.parametrize("shape,match", [
    ((-1, 4, 2, 1, 1), "batch"), ((65536, 4, 2, 1, 1), "batch"), ((2, 0, 2, 1, 1), "max_pages"), ((2, 16385, 2, 1, 1), "max_pages"),
    ((2, 4, 0, 0, 1), "keep"), ((2, 4, 2, 2, 1), "keep"), ((2, 4, 2, -1, 1), "keep"), ((2, 4, 2, 1, 0), "keep"),
    ((2, 4, 4097, 1, 1), "keep"), ((2, 4, 2, 2 ** 31 - 1, 2 ** 31 - 1), "keep")])
def test_bad_shapes_are_refused(shape, match):
    select(shape=shape, match=match)


def test_other_refusals():
    for name in ("pages", "lengths", "out", "held"):
        select(**{name: None}, match="null")
        select(**{name: FAR[5] + 2}, match="unaligned")
    select(blocks=FAR[5] + 1, match="unaligned")
    select(status=FAR[5] + 1, match="unaligned")
    select(q=heads(n=12), match="multiple")
    select(q=heads(n=8 * 65), match="64 times")
    select(q=heads(n=32, dtype=3), match="type")
    select(q=heads(n=32, data=None), match="null")
    # lists of 2 x 8 x 2 entries, a table of 2 x 4, lengths of 2
    select(held=FAR[1] + 4, match="overlap")
    select(held=FAR[1], match="overlap")
    select(out=FAR[0] - 124, match="overlap")
    select(blocks=FAR[2] + 124, match="overlap")
    select(blocks=FAR[3] - 4, match="overlap")
    refused(ops.wici_kv_bounds_update, 0, cache(), bounds(), None, 1, match="null")
    refused(ops.wici_kv_bounds_update, 0, cache(), bounds(), A + 2, 1, match="unaligned")
    refused(ops.wici_kv_bounds_update, 0, cache(), bounds(), A, -1, match="count")
    refused(ops.wici_kv_bounds_update, 0, cache(), bounds(), A, 1 << 27, match="count")
    shape = ops.wici_attn_shape(1, 4, 5, 0.1)
    refused(ops.wici_selected_attention, 0, cache(), shape, A, A, heads(n=32), heads(n=32), None, A, match="window")
    refused(ops.wici_selected_attention, 0, cache(), ops.wici_attn_shape(1, 0, 0, 0.1), A, A, heads(n=32), heads(n=32), None, A, match="max_pages")


def test_calls_without_work_touch_nothing():
    ops.wici_kv_bounds_update(0, cache(), bounds(), None, 0)
    ops.wici_kv_select(0, cache(), bounds(), ops.wici_select_shape(0, 4, 2, 1, 1), None, None, heads(n=32, data=None), None, None)


def test_tensors_are_checked_by_the_binding():
    torch = pytest.importorskip("torch")
    kv = object.__new__(ops.PagedKV)                           # without a device: only what the checks look at
    kv.n_kv_heads, kv.head_dim, kv.n_pages, kv.device = 2, 64, 3, torch.device("cpu")
    kv.cache = cache(kv=2, d=64, pages=3)
    record = ops.wici_kv_bounds_bytes(2, 64)
    for data in (torch.zeros(3 * record + 16, dtype=torch.uint8), torch.zeros(3 * record, dtype=torch.int8),
                 torch.zeros(6 * record, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="data"):
            ops.KeyBounds(kv, data=data)
    b = ops.KeyBounds(kv)
    assert b.codes.shape == (3, 2, 2, 64) and b.scales.shape == (3, 2) and b.data.numel() == 3 * record
    assert b.codes.data_ptr() == b.data.data_ptr() and b.scales.data_ptr() == b.data.data_ptr() + 256


def test_oracle_scores_are_the_largest_products_within_the_bounds():
    rng = np.random.default_rng(0)
    k = rng.normal(size=(16, 32)).astype(np.float32)
    codes, scale = paged.key_bounds(k)
    assert codes.min() >= -127 and codes.max() <= 127 and scale == np.abs(k).max() * (np.float32(1) / np.float32(127))
    q = rng.normal(size=(3, 32)).astype(np.float32)
    s = paged.page_scores(q, codes[None], [scale])[0] / 1023
    ends = codes.astype(np.float64) * scale
    want = max(np.maximum(x * ends[0], x * ends[1]).sum() for x in q.astype(np.float64))
    assert abs(s - want) < 32 * np.abs(q).max() / 1023 * np.abs(k).max()
    assert s >= (q @ k.T).max() - np.abs(q).sum(1).max() * scale - 32 * np.abs(q).max() / 1023 * np.abs(k).max()


def test_oracle_selection():
    s = np.array([5, 1, 3, 3, 9, 3, 0, 2], np.float32)
    assert paged.selected_pages(s, 8, 1, 1) == list(range(8))
    assert paged.selected_pages(s, 4, 1, 1) == [0, 2, 4, 7]
    assert paged.selected_pages(s, 4, 0, 1) == [0, 2, 4, 7]
    assert paged.selected_pages(s, 3, 1, 2) == [0, 6, 7]
    assert paged.selected_pages(s, 5, 0, 1) == [0, 2, 3, 4, 7]
    assert np.isnan(paged.key_bounds(np.array([[1.0, np.inf]]))[1]) and paged.key_bounds(np.zeros((2, 4)))[1] == 0


@pytest.mark.parametrize("out", ["out", "held", "blocks"])
def test_outputs_over_what_a_selection_reads_are_refused(out):
    def places(q=FAR[5], b=FAR[6], c=FAR[7], status=None):
        return dict(q=heads(n=32, data=q), b=bounds(data=b), c=cache(data=c), status=status)
    n = 8 if out == "held" else 128                            # bytes of the output
    q_bytes, record, page = 2 * 32 * 128 * 2, ops.wici_kv_bounds_bytes(8, 128), cache().page_stride
    for at, size in ((FAR[5], q_bytes), (FAR[6], 4 * record), (FAR[7], 4 * page)):
        for first in (at - n + 4, at, at + size - 4):
            select(**{out: first}, **places(), match="overlap")
    word = A + (1 << 36)
    for first in (word - n + 4, word):
        select(**{out: first}, **places(status=word), match="overlap")
    # inside a record of records that lie apart, and a head of heads that do
    select(**{out: FAR[6] + 3 * (1 << 16) + 64}, **dict(places(), b=bounds(data=FAR[6], stride=1 << 16)), match="overlap")
    at = A + (1 << 37)
    apart = heads(n=32, data=at, token=1 << 20, head=1 << 12)
    select(**{out: at + 2 * ((1 << 20) + 31 * (1 << 12)) + 64}, **dict(places(), q=apart), match="overlap")
