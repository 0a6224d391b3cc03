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
