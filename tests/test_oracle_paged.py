"""Pins of the paged operators' oracle (oracle/paged.py): no GPU."""
import numpy as np
import pytest

from oracle import llama, paged

torch = pytest.importorskip("torch")


def test_e4m3_table_and_rounding_agree_with_torch():
    every = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(every, paged.E4M3)
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.normal(size=20000) * 2.0 ** rng.integers(-12, 9, 20000), every[np.isfinite(every)],
                        (paged.E4M3[:126] + paged.E4M3[1:127]) / 2, -(paged.E4M3[:126] + paged.E4M3[1:127]) / 2])
    v = np.clip(v, -448, 448).astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(paged.e4m3_codes(v), want)


def test_unscaled_half_rope_is_the_model_oracles():
    x = np.random.default_rng(1).normal(size=(5, 3, 64))
    pos = np.array([0, 1, 7, 1000, 131071])
    f, g = paged.rope_frequencies(64, 5e5)
    want = llama.apply_rope(x, *llama.rope_cos_sin(pos, 64, 5e5))
    np.testing.assert_allclose(paged.rope(x, pos, 64, f, g), want, rtol=0, atol=1e-12)


def test_interleaved_rope_is_complex_multiplication_and_inverse_undoes_it():
    x = np.random.default_rng(2).normal(size=(4, 2, 32))
    pos = np.array([3, 0, 12, -5])
    f, _ = paged.rope_frequencies(16, 1e4)
    y = paged.rope(x, pos, 16, f, interleaved=True)
    z = (x[..., 0:16:2] + 1j * x[..., 1:16:2]) * np.exp(1j * pos[:, None] * f)[:, None]
    np.testing.assert_allclose(y[..., 0:16:2], z.real, atol=1e-12)
    np.testing.assert_allclose(y[..., 1:16:2], z.imag, atol=1e-12)
    np.testing.assert_array_equal(y[..., 16:], x[..., 16:])
    np.testing.assert_allclose(paged.rope(y, pos, 16, f, interleaved=True, inverse=True), x, atol=1e-12)


def test_scaling_rules_at_their_ends():
    f, _ = paged.rope_frequencies(128, 5e5)
    lin, _ = paged.rope_frequencies(128, 5e5, "linear", 4.0)
    np.testing.assert_allclose(lin, f / 4)
    b, _ = paged.rope_frequencies(128, 5e5, "bands", 8.0, 8192, 1.0, 4.0)
    wave = 2 * np.pi / f
    assert np.array_equal(b[wave < 8192 / 4], f[wave < 8192 / 4])
    np.testing.assert_allclose(b[wave > 8192], f[wave > 8192] / 8)
    between = (wave > 8192 / 4) & (wave < 8192)
    assert between.any() and np.all((b[between] < f[between]) & (b[between] > f[between] / 8))
    y, g = paged.rope_frequencies(128, 5e5, "yarn", 8.0, 8192, 1.0, 32.0)
    assert y[0] == f[0] and np.isclose(y[-1], f[-1] / 8) and np.isclose(g, 1 + 0.1 * np.log(8))
    assert np.all(np.diff(y) < 0)


@pytest.mark.parametrize("fmt,half_step", [("int8", 0.5 / 127), ("e4m3", 2.0 ** -4)])
def test_quantised_heads_are_within_half_a_step(fmt, half_step):
    x = np.random.default_rng(3).normal(size=(50, 64))
    x[7] = 0
    x[9, 3] = np.inf
    codes, scales = paged.quantise(x, fmt)
    got = paged.code_values(codes, fmt) * scales[:, None]
    assert np.all(np.isnan(got[9])) and np.all(got[7] == 0)
    ok = [i for i in range(50) if i != 9]
    top = np.abs(x[ok]).max(-1, keepdims=True)
    bound = half_step * (top if fmt == "int8" else np.maximum(np.abs(x[ok]), top / 448 * 2.0 ** -6))
    assert np.all(np.abs(got[ok] - x[ok]) <= bound * (1 + 1e-12))


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_pack_and_unpack(fmt):
    rng = np.random.default_rng(4)
    codes = rng.integers(0, 256, size=(48, 2, 3, 64))
    codes = codes.astype(np.uint16) if fmt == "bf16" else codes.astype(np.uint8).view(np.int8 if fmt == "int8" else np.uint8)
    scales = None if fmt == "bf16" else rng.normal(size=(48, 2, 3)).astype(np.float32)
    data = paged.pack(codes, scales, fmt)
    assert data.size == 3 * 2 * 3 * paged.block_bytes(fmt, 64)
    c, s = paged.unpack(data, 3, 64, fmt)
    np.testing.assert_array_equal(c, codes)
    if scales is not None:
        np.testing.assert_array_equal(s, scales)
        # the place of one token by hand: slot 21 = page 1, place 5; V of head 2
        block = data[(1 * 6 + 1 * 3 + 2) * paged.block_bytes(fmt, 64):]
        np.testing.assert_array_equal(block[5 * 64:6 * 64].view(codes.dtype), codes[21, 1, 2])
        assert block[16 * 64 + 20:16 * 64 + 24].view(np.float32)[0] == scales[21, 1, 2]


def test_attention_against_dense_softmax():
    rng = np.random.default_rng(5)
    q, k, v = rng.normal(size=(2, 4, 32)), rng.normal(size=(64, 2, 32)), rng.normal(size=(64, 2, 32))
    pages = np.array([[2, 0, 3], [1, 3, 2]])
    out, lse, _ = paged.paged_attention(q, k, v, pages, [37, 0], 0.3)
    assert np.all(out[1] == 0) and np.all(lse[1] == -np.inf)
    order = np.concatenate([np.arange(32, 48), np.arange(16), np.arange(48, 64)])[:37]
    for h in range(4):
        s = torch.from_numpy(k[order, h // 2] @ q[0, h] * 0.3)
        want = torch.softmax(s, 0).numpy() @ v[order, h // 2]
        np.testing.assert_allclose(out[0, h], want, atol=1e-13)
        assert np.isclose(lse[0, h], torch.logsumexp(s, 0).item())
    win, _, _ = paged.paged_attention(q, k, v, pages, [37, 0], 0.3, window=5)
    last, _, _ = paged.paged_attention(q[:1], k[order[-5:]], v[order[-5:]], [[0]], [5], 0.3)
    np.testing.assert_allclose(win[0], last[0], atol=1e-13)
