"""Attention of the batched decode step where queries, keys and the scale are far from 1: large logits, and factors near the
ends of fp32's range whose product is an ordinary logit.

Tolerances as in tests/test_gpu_ops.py.  Where the largest logit is 10% of itself above the others' and that is more than
a hundred, the other keys' weights are below 2^-126 in base 2 and count as 0: the result is that key's value, its one
weight divided by itself (in two terms: 2^-16 as there)."""
import numpy as np
import pytest

from oracle import paged

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2608_24204_gb300 import PagedKV  # noqa: E402
from tests.test_gpu_ops import DT, check_attention, f64, half_step, ints, randn, within  # noqa: E402


def stored(k, v, fmt):
    """A cache of the tokens in order, and its values by slot."""
    n, kv, d = k.shape
    pages = n // 16 + 1
    cache = PagedKV(kv, d, fmt, n_pages=pages)
    cache.append(k, v, ints(range(n)))
    vals = np.zeros((16 * pages, 2, kv, d))
    for which, t in enumerate(cache.read(ints(range(n)), dtype=torch.float32)):
        vals[:n, which] = f64(t)
    return cache, vals, np.arange(pages)[None]


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3", "e2m1"])
@pytest.mark.parametrize("dtype,group,d", [("bf16", 4, 128), ("f32", 3, 64), ("f32", 5, 128), ("bf16", 12, 64)])
@pytest.mark.parametrize("q_size,k_size,scale", [(0, 30, 1.0), (10, 20, -1.0), (0, 40, 0.3), (-20, 90, 0.7), (40, 40, 1.0), (-60, 60, 2.0 ** 30)])
def test_large_logits(fmt, dtype, group, d, q_size, k_size, scale):
    # every key is a multiple of one direction, the largest and the smallest multiple one key's alone
    rng = np.random.default_rng(d + group + k_size)
    n = 200
    along = rng.choice([-1.0, 1.0], d) * rng.uniform(1, 2, d)
    times = rng.uniform(-0.7, 0.7, n)
    times[[137, 60]] = 1.0, -1.0
    k = torch.tensor(times[:, None, None] * along * 2.0 ** k_size, device="cuda").to(DT[dtype])
    q = torch.tensor((rng.uniform(0.5, 1, group) * rng.choice([-1.0, 1.0], group))[None, :, None] * along * 2.0 ** q_size, device="cuda").to(DT[dtype])
    cache, vals, pages = stored(k, randn(rng, n, 1, d, dtype=dtype), fmt)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = cache.attend(q, ints(pages), ints([n]), scale=scale, out=torch.empty(q.shape, device="cuda"), lse=lse)
    scale = float(np.float32(scale))
    logits = f64(q)[0] @ vals[:n, 0, 0].T * scale
    best = logits.argmax(1)
    rest = logits.copy()
    rest[np.arange(group), best] = -np.inf
    assert np.all(logits.max(1) - rest.max(1) > np.maximum(0.1 * logits.max(1), 100.0))
    want = vals[best, 1, 0]
    within(f64(out[0]), want, 2.0 ** -16 * np.abs(want) + half_step(want, "f32"), "out")
    size = np.abs(f64(q)[0]) @ np.abs(vals[:n, 0, 0]).T * abs(scale)
    within(f64(lse[0]), logits.max(1), size.max(1) * (2 * d * 2.0 ** -23 + 2.0 ** -16) + 2.0 ** -20, "lse")
