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


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype,group,d", [("bf16", 4, 128), ("f32", 3, 64), ("bf16", 12, 64)])
@pytest.mark.parametrize("q_size,k_size,scale", [(-110, 110, 1.0), (-100, 125, 2.0 ** -22), (0, 110, 2.0 ** -110), (-20, 118, -2.0 ** -98),
                                                  (-115, 107, 1.0), (-120, 122, 0.088), (-125, 126, 0.088), (100, -80, 2.0 ** -15), (120, -85, 2.0 ** -30)])
def test_keys_of_any_size(fmt, dtype, group, d, q_size, k_size, scale):
    """Keys and queries near the ends of what fp32 holds, whose logits the other or the scale makes ordinary ones."""
    check_moderate(fmt, dtype, group, d, q_size, k_size, scale)


def check_moderate(fmt, dtype, group, d, q_size, k_size, scale):
    rng = np.random.default_rng(abs(d + group + k_size))
    n = 150
    # below 4 2^k_size: finite numbers, of the products' sums as well
    k = torch.tensor(np.clip(rng.normal(size=(n, 1, d)), -4, 4) * 2.0 ** k_size * d ** -0.5, device="cuda").to(DT[dtype])
    q = torch.tensor(rng.normal(size=(2, group, d)) * 2.0 ** q_size, device="cuda").to(DT[dtype])
    cache, vals, pages = stored(k, randn(rng, n, 1, d, dtype=dtype), fmt)
    lse = torch.empty(q.shape[:2], device="cuda")
    pages, lengths = np.repeat(pages, 2, 0), [n, 77]
    out = cache.attend(q, ints(pages), ints(lengths), scale=scale, out=torch.empty(q.shape, device="cuda"), lse=lse)
    stored_as = (paged.unpack_e2m1 if fmt == "e2m1" else lambda *x: paged.unpack(*x, fmt))(cache.data.cpu().numpy(), 1, d)
    v_scales = stored_as[-1][:n, 1, 0].astype(np.float64)
    scale, q64 = float(np.float32(scale)), f64(q)
    want, want_lse, weight = paged.paged_attention(q64, vals[:, 0], vals[:, 1], pages, lengths, scale)
    for b, m in enumerate(lengths):
        keys, v, s = vals[:m, 0, 0], vals[:m, 1, 0], v_scales[:m]
        for h in range(group):
            # the terms of check_attention, and one for logits far apart: a key's weight times its scale of V is held to 2^-32
            # of the largest such product, and what is lost of it counts v / scale times
            p = np.exp(keys @ q64[b, h] * scale - want_lse[b, h])
            ds = float(np.max(np.abs(keys) @ np.abs(q64[b, h])) * abs(scale)) * (2 * d * 2.0 ** -23 + (2.0 ** -16 if dtype == "f32" else 0.0))
            rel = 2 * ds + 2.0 ** -16 + 2.0 ** -21 + m * 2.0 ** -23
            small = 2.0 ** -32 * (p * s).max() * (np.abs(v) / s[:, None]).sum(0)
            within(f64(out[b, h]), want[b, h], rel * weight[b, h] + small * (1 + rel) + half_step(want[b, h], "f32"), "out")
            within(float(lse[b, h]), want_lse[b, h], ds + 2.0 ** -20 + m * 2.0 ** -23 + 2.0 ** -23 * abs(want_lse[b, h]), "lse")


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype,group,d", [("bf16", 4, 128), ("f32", 3, 64)])
@pytest.mark.parametrize("q_size,k_size", [(1e-33, 1e33), (1e-35, 1e35), (3e-4, 3e35)])
def test_every_element_of_a_key_is_large(fmt, dtype, group, d, q_size, k_size):
    """Sums over the head of 2^20 and more times a key's scale, before the query's own size comes in."""
    n = 40
    k = torch.tensor(np.cos(np.arange(n))[:, None, None] * np.full((n, 1, d), k_size), device="cuda").to(DT[dtype])
    q = torch.full((1, group, d), q_size, device="cuda").to(DT[dtype])
    cache, vals, pages = stored(k, randn(np.random.default_rng(d), n, 1, d, dtype=dtype), fmt)
    lse = torch.empty(q.shape[:2], device="cuda")
    scale = float(np.float32(1e-33 / (q_size * (k_size / 1e33)) * d ** -0.5))
    out = cache.attend(q, ints(pages), ints([n]), scale=scale, out=torch.empty(q.shape, device="cuda"), lse=lse)
    check_attention(cache, q, pages, [n], vals, scale, 0, out, lse, dtype, "f32")


@pytest.mark.parametrize("d", [64, 128])
def test_long_fp32_sums_are_not_all_cut_the_same_way(d):
    """The mean relative error of positive results over long runs of keys.  Additions on tensor cores are cut, by 2^-23 of the sum at
    most: 8 of a unit's 64 keys (head_dim 64) make 2^-20 of it; what is rounded to the nearest averages out over the 4096
    elements, of which each row's sum of weights is common to head_dim: some 400 additions of 2^-25 each in 8 x 20 lanes of 64
    rows, 6e-9."""
    n, kv, group, batch = 1 << 18, 8, 4, 2
    g = torch.Generator(device="cuda").manual_seed(d)
    cache = PagedKV(kv, d, "e2m1", n_pages=batch * n // 16)
    slots = torch.arange(batch * n, device="cuda", dtype=torch.int32)
    for i in range(0, batch * n, n // 4):
        at = slots[i:i + n // 4]
        k = torch.randn(len(at), kv, d, generator=g, device="cuda")
        cache.append(k, torch.rand(len(at), kv, d, generator=g, device="cuda") + 0.5, at)
    q = torch.randn(batch, kv * group, d, generator=g, device="cuda")
    pages = torch.arange(batch * n // 16, device="cuda", dtype=torch.int32).view(batch, -1)
    out = cache.attend(q, pages, ints([n, n]), scale=0.25 * d ** -0.5)
    cache.check()
    off = []
    for b in range(batch):
        k, v = cache.read(slots[b * n:(b + 1) * n], dtype=torch.float32)
        for h in range(kv):
            p = torch.softmax(q[b, h * group:(h + 1) * group].double() @ k[:, h].double().T * (0.25 * d ** -0.5), -1)
            want = p @ v[:, h].double()
            off.append((out[b, h * group:(h + 1) * group].double() / want - 1).mean())
    assert abs(torch.stack(off).mean().item()) < 2.0 ** -20 + 2.0 ** -21


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3", "e2m1"])
@pytest.mark.parametrize("dtype,group,d", [("bf16", 4, 128), ("f32", 3, 64), ("bf16", 12, 64)])
def test_queries_of_zeros_beside_a_large_scale(fmt, dtype, group, d):
    # its logits are 0 whatever the scale and the keys are, as far as these are finite
    n = 90
    rng = np.random.default_rng(d)
    k = torch.tensor(rng.normal(size=(n, 1, d)) * 2.0 ** 100, device="cuda").to(DT[dtype])
    cache, vals, pages = stored(k, randn(rng, n, 1, d, dtype=dtype), fmt)
    q = torch.zeros(1, group, d, dtype=DT[dtype], device="cuda")
    lse = torch.empty(1, group, device="cuda")
    out = cache.attend(q, ints(pages), ints([n]), scale=2.0 ** 60, out=torch.empty(1, group, d, device="cuda"), lse=lse)
    check_attention(cache, q, pages, [n], vals, 2.0 ** 60, 0, out, lse, dtype, "f32")
