"""Host-side checks of include/wici_ops.h and its binding that need no GPU: the exports, the
rope plan, page sizes, and every refusal (arguments are checked before a device is touched)."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import paged
from paper_2608_24204_gb300 import build, ops, wici

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                                     # an aligned address that nothing dereferences


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def heads(n=8, d=128, dtype=ops.WICI_BF16, data=A, token=None, head=None):
    return ops.wici_heads(data, n * d if token is None else token, d if head is None else head, n, dtype)


def cache(fmt=ops.WICI_KV_BF16, kv=8, d=128, pages=4, data=A, stride=None):
    return ops.wici_kv_cache(data, ops.wici_kv_page_bytes(fmt, kv, d) if stride is None else stride, pages, kv, d, fmt)


def plan(d=128, rot=None, **kw):
    return ops.Rope(d, 5e5, rot_dim=rot, **kw).plan


def refused(f, *args, match=""):
    with pytest.raises(wici.WiciError) as e:
        f(*args)
    assert e.value.status == wici.WICI_E_ARG
    assert match in str(e.value), str(e.value)


def test_exports_are_the_headers():
    with open(os.path.join(ROOT, "include", "wici_ops.h")) as f:
        names = sorted(set(re.findall(r"^(?:int|int64_t) (wici_\w+)\(", f.read(), re.M)))
    assert names == sorted(ops.EXPORTS)
    for n in names:
        assert hasattr(ops.lib(), n)


@pytest.mark.parametrize("d,rot,scaling", [(128, 128, "none"), (64, 32, "linear"), (128, 128, "bands"), (80, 20, "yarn"),
                                           (256, 256, "yarn"), (2, 2, "none")])
def test_plan_holds_the_frequencies_as_turns(d, rot, scaling):
    kw = {} if scaling == "none" else {"factor": 8.0, "original_len": 8192, "low": 1.0, "high": 4.0}
    p = ops.Rope(d, 5e5, rot_dim=rot, scaling=scaling, **kw).plan
    f, g = paged.rope_frequencies(rot, 5e5, scaling, **({} if scaling == "none" else kw))
    got = np.array([float(t) for t in p.turns[:rot // 2]]) * 2 * np.pi / 2.0 ** 64
    # double arithmetic of pow and the rule: a few 2^-52; a turn is stored to the nearest 2^-63: 2^-64 turns off
    np.testing.assert_allclose(got, f, rtol=1e-13, atol=2.0 ** -64 * 2 * np.pi)
    assert all(t == 0 for t in p.turns[rot // 2:])
    assert p.gain == np.float32(g) and (p.head_dim, p.rot_dim, p.interleaved) == (d, rot, 0)
    assert ops.Rope(d, 5e5, rot_dim=rot, scaling=scaling, gain=1.5, **kw).plan.gain == 1.5


@pytest.mark.parametrize("kw,match", [
    ({"head_dim": 258}, "head_dim"), ({"head_dim": 63}, "head_dim"), ({"rot_dim": 130}, "rot_dim"),
    ({"rot_dim": 3}, "rot_dim"), ({"rot_dim": 0}, "rot_dim"), ({"theta": 1.0}, "theta"), ({"theta": float("nan")}, "theta"),
    ({"factor": 2.0}, "factor"), ({"factor": 0.5, "scaling": "linear"}, "factor"),
    ({"scaling": "bands", "factor": 8.0, "low": 4.0, "high": 1.0, "original_len": 10}, "low"),
    ({"scaling": "yarn", "factor": 8.0, "low": 1.0, "high": 32.0, "original_len": 0}, "original_len"),
    ({"gain": -1.0}, "gain"), ({"gain": float("inf")}, "gain")])
def test_bad_ropes_are_refused(kw, match):
    refused(lambda: ops.Rope(**{"head_dim": 128, "theta": 1e4, **kw}), match=match)
    with pytest.raises(ValueError):
        ops.Rope(128, 1e4, scaling="no such rule")


def test_page_bytes():
    assert ops.wici_kv_page_bytes(ops.WICI_KV_BF16, 8, 128) == 2 * 8 * 16 * 128 * 2
    assert ops.wici_kv_page_bytes(ops.WICI_KV_INT8, 3, 64) == 2 * 3 * 16 * (64 + 4)
    assert ops.wici_kv_page_bytes(ops.WICI_KV_E4M3, 1, 128) == 2 * paged.block_bytes("e4m3", 128)
    assert ops.wici_kv_page_bytes(9, 8, 128) == ops.wici_kv_page_bytes(0, 8, 96) == ops.wici_kv_page_bytes(0, 0, 64) == 0


BAD_TENSORS = [
    (heads(data=None), "null"), (heads(data=A + 1), "unaligned"), (heads(dtype=3), "type"), (heads(n=0), "heads"),
    (heads(token=-1), "stride"), (heads(head=-128), "stride"), (heads(token=1 << 62), "stride")]


@pytest.mark.parametrize("bad,match", BAD_TENSORS)
def test_bad_tensors_are_refused(bad, match):
    good = heads()
    refused(ops.wici_rope, 0, plan(), 0, A, 5, bad, good, match=match)
    refused(ops.wici_rope, 0, plan(), 0, A, 5, good, bad, match=match)
    refused(ops.wici_kv_append, 0, cache(), A, 5, bad, good, match=match)
    refused(ops.wici_kv_append, 0, cache(), A, 5, good, bad, match=match)
    refused(ops.wici_kv_read, 0, cache(), A, 5, bad, None, match=match)
    shape = ops.wici_attn_shape(5, 4, 0, 0.1)
    refused(ops.wici_paged_attention, 0, cache(), shape, A, A, bad, good, None, A, match=match)
    refused(ops.wici_paged_attention, 0, cache(), shape, A, A, good, bad, None, A, match=match)


@pytest.mark.parametrize("out", [heads(head=64), heads(token=512), heads(token=0), heads(token=128, head=128 * 4)])
def test_outputs_whose_heads_share_places_are_refused(out):
    refused(ops.wici_rope, 0, plan(), 0, A, 5, heads(), out, match="overlap")
    refused(ops.wici_kv_read, 0, cache(), A, 5, None, out, match="overlap")
    refused(ops.wici_paged_attention, 0, cache(), ops.wici_attn_shape(5, 4, 0, 0.1), A, A, heads(), out, None, A,
            match="overlap")


@pytest.mark.parametrize("bad,match", [
    (cache(data=None), "null"), (cache(data=A + 8), "aligned"), (cache(pages=0), "n_pages"), (cache(pages=1 << 27), "n_pages"),
    (cache(stride=2 * 8 * 4096 - 16), "page_stride"), (cache(stride=2 * 8 * 4096 + 8), "page_stride"),
    (ops.wici_kv_cache(A, 1 << 20, 4, 8, 96, 0), "head_dim"), (ops.wici_kv_cache(A, 1 << 20, 4, 0, 64, 0), "n_kv_heads"),
    (ops.wici_kv_cache(A, 1 << 20, 4, 8, 64, 3), "format"), (ops.wici_kv_cache(A, 1 << 20, 4, 1025, 64, 0), "n_kv_heads")])
def test_bad_caches_are_refused(bad, match):
    n = max(bad.n_kv_heads, 1)
    t = heads(n=n, d=128)
    refused(ops.wici_kv_append, 0, bad, A, 1, t, t, match=match)
    refused(ops.wici_kv_read, 0, bad, A, 1, t, t, match=match)
    refused(ops.wici_paged_attention, 0, bad, ops.wici_attn_shape(1, 4, 0, 0.1), A, A, t, t, None, A, match=match)
    refused(ops.wici_paged_attention_workspace_bytes, bad, n, 1, match=match)


def test_other_refusals():
    h, h4, f32 = heads(), heads(n=4), heads(dtype=ops.WICI_F32)
    refused(ops.wici_rope, 0, plan(), 2, A, 1, h, h, match="inverse")
    refused(ops.wici_rope, 0, plan(), 0, None, 1, h, h, match="positions")
    refused(ops.wici_rope, 0, plan(), 0, A, -1, h, h, match="tokens")
    refused(ops.wici_rope, 0, plan(), 0, A, 1 << 31, h, h, match="tokens")
    refused(ops.wici_rope, 0, plan(), 0, A, 1, h, h4, match="differ")
    refused(ops.wici_rope, 0, plan(), 0, A, 1, h, f32, match="differ")
    refused(ops.wici_rope, 0, ops.wici_rope_plan(), 0, A, 1, h, h, match="plan")
    c = cache()
    refused(ops.wici_kv_append, 0, c, None, 1, h, h, match="slots")
    refused(ops.wici_kv_append, 0, c, A, 1, h4, h4, match="heads")
    refused(ops.wici_kv_append, 0, c, A, 1, h, f32, match="type")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, None, A, match="rope")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, None, None, h, h, match="rope")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, plan(), A, h, None, match="together")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, plan(), None, match="positions")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, plan(64), A, match="head_dim")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, plan(128, 24), A, match="multiple of 16")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, plan(), A, h, h4, match="heads")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, plan(), A, f32, f32, match="type")
    refused(ops.wici_kv_read, 0, c, A, 1, None, None, match="neither")
    refused(ops.wici_kv_read, 0, c, None, 1, h, h, match="slots")
    refused(ops.wici_kv_read, 0, c, A, 1, h, f32, match="type")
    refused(ops.wici_kv_read, 0, c, A, 1, h4, None, match="heads")

    def attention(shape=(1, 4, 0, 0.1), pages=A, lengths=A, q=h, out=h, ws=A, match=""):
        refused(ops.wici_paged_attention, 0, c, ops.wici_attn_shape(*shape), pages, lengths, q, out, None, ws, match=match)

    attention(shape=(-1, 4, 0, 0.1), match="batch")
    attention(shape=(65536, 4, 0, 0.1), match="batch")
    attention(shape=(1, 0, 0, 0.1), match="max_pages")
    attention(shape=(1, 1 << 27, 0, 0.1), match="max_pages")
    attention(shape=(1, 4, -1, 0.1), match="window")
    attention(shape=(1, 4, 0, float("nan")), match="scale")
    attention(shape=(1, 4, 0, float("inf")), match="scale")
    attention(pages=None, match="pages")
    attention(lengths=None, match="lengths")
    attention(ws=None, match="workspace")
    attention(ws=A + 4, match="workspace")
    attention(q=h, out=heads(n=16), match="differ")
    attention(q=heads(n=12), out=heads(n=12), match="multiple")
    refused(ops.wici_paged_attention_workspace_bytes, c, 12, 1, match="multiple")
    refused(ops.wici_paged_attention_workspace_bytes, c, 8, -1, match="batch")
    assert ops.lib().wici_paged_attention_workspace_bytes(c, 8, 1, None) == wici.WICI_E_ARG
    assert ops.lib().wici_rope_make_plan(None, None) == wici.WICI_E_ARG
    assert ops.lib().wici_paged_attention(0, c, None, A, A, h, h, None, A, None) == wici.WICI_E_ARG
    n = ctypes.c_int32()
    assert ops.lib().wici_kv_view(None, 0, c, ctypes.c_void_p(), n) == wici.WICI_E_ARG


def test_empty_calls_need_no_device():
    h, none = heads(), heads(data=None)
    ops.wici_rope(0, plan(), 0, None, 0, none, none)
    ops.wici_kv_append(0, cache(), None, 0, none, none)
    ops.wici_kv_read(0, cache(), None, 0, h, None)
    ops.wici_paged_attention(0, cache(), ops.wici_attn_shape(0, 4, 0, 0.1), None, None, none, none, None, None)


def test_workspace_grows_with_the_batch():
    sizes = [ops.wici_paged_attention_workspace_bytes(cache(), 32, b) for b in (0, 1, 64, 65535)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_tensors_on_the_cpu_or_of_a_wrong_kind_are_refused():
    import torch
    r = ops.Rope(64, 1e4)
    x, pos = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        r.apply(x, pos)
    kv = ops.PagedKV(2, 64, "int8", n_pages=2, device="cpu")
    assert kv.data.numel() == 2 * 2 * 2 * 16 * 68
    with pytest.raises(ValueError, match="CUDA"):
        kv.append(x, x, pos)
    with pytest.raises(ValueError, match="CUDA"):
        kv.read(pos)
    with pytest.raises(ValueError, match="CUDA"):
        kv.attend(x, torch.zeros(3, 1, dtype=torch.int32), pos)
    for bad in (torch.zeros(3, 64), torch.zeros(3, 2, 32)):
        with pytest.raises(ValueError, match="expected"):
            ops.heads_of(bad, 64, bad.device, "x")
    with pytest.raises(TypeError):
        ops.heads_of(x.double(), 64, x.device, "x")
    with pytest.raises(ValueError, match="adjacent"):
        ops.heads_of(torch.zeros(3, 64, 2).transpose(1, 2), 64, x.device, "x")
    for kw in ({"fmt": "int4", "n_pages": 1}, {"head_dim": 96, "n_pages": 1}, {"n_pages": None},
               {"data": torch.zeros(100, dtype=torch.uint8)}, {"data": torch.zeros(8192)}):
        with pytest.raises(ValueError):
            ops.PagedKV(**{"n_kv_heads": 2, "head_dim": 64, "device": "cpu", **kw})


@pytest.mark.parametrize("off", [1, 2, 3])
def test_unaligned_words_are_refused(off):
    h, c, u = heads(), cache(), A + off
    refused(ops.wici_rope, 0, plan(), 0, u, 1, h, h, match="unaligned")
    refused(ops.wici_kv_append, 0, c, u, 1, h, h, match="unaligned")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, plan(), u, match="unaligned")
    refused(ops.wici_kv_append, 0, c, A, 1, h, h, None, None, None, None, u, match="unaligned")
    refused(ops.wici_kv_read, 0, c, u, 1, h, h, match="unaligned")
    refused(ops.wici_kv_read, 0, c, A, 1, h, h, u, match="unaligned")
    shape = ops.wici_attn_shape(1, 4, 0, 0.1)
    for i in range(4):
        pages, lengths, lse, status = (u if i == j else A for j in range(4))
        refused(ops.wici_paged_attention, 0, c, shape, pages, lengths, h, h, lse, A, status, match="unaligned")


def test_more_pages_than_a_launch_can_count_are_refused():
    h = heads(n=64)
    refused(ops.wici_paged_attention, 0, cache(), ops.wici_attn_shape(1, (1 << 25) - 2, 0, 0.1), A, A, h, h, None, A,
            match="2^31")


def test_the_header_is_c(tmp_path):
    import shutil
    import subprocess
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("needs gcc")
    src = tmp_path / "t.c"
    src.write_text(f'#include "{ROOT}/include/wici_ops.h"\n_Static_assert(sizeof(wici_heads) == 32, "");\n'
                   '_Static_assert(sizeof(wici_rope_plan) == 1040, "");\n_Static_assert(sizeof(wici_kv_cache) == 32, "");\n'
                   '_Static_assert(sizeof(wici_attn_shape) == 16, "");\n_Static_assert(sizeof(wici_rope_spec) == 64, "");\n')
    subprocess.run([cc, "-std=c11", "-Wall", "-Werror", "-fsyntax-only", str(src)], check=True)
    assert [ctypes.sizeof(t) for t in (ops.wici_heads, ops.wici_rope_plan, ops.wici_kv_cache, ops.wici_attn_shape,
                                       ops.wici_rope_spec)] == [32, 1040, 32, 16, 64]


def test_every_rows_block_holds_its_tokens(tmp_path):
    # the shape of a row-wise launch (csrc/ops.h) for every rotation, head and token count: a row for each token of a
    # block, whole warps for the shuffles of a cache row, and no more threads than the kernels are compiled for
    import shutil
    import subprocess
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("needs g++")
    src, exe = tmp_path / "t.cc", tmp_path / "t"
    src.write_text(f'#include "{ROOT}/paper_2608_24204_gb300/csrc/ops.h"\n' + r"""
#include <cstdio>
#include <initializer_list>
using namespace wici;
int main() {
    int most = 0;
    for (int64_t tokens : {1, 100, 4863, 4864, 9727, 9728, 19455, 19456, 1000000})
        for (int heads : {1, 2, 3, 7, 40, 1000})
            for (int sms : {1, 20, 152, 200})
                for (int chunks = 1; chunks <= 17; ++chunks) {
                    const RowBlock b = row_block(tokens, heads, chunks, sms);
                    const bool power = b.tokens > 0 && (b.tokens & (b.tokens - 1)) == 0;
                    const bool cache = chunks == 4 || chunks == 8;      // of 64 and 128 elements
                    if (!power || b.tokens > kBlockTokens || b.rows < b.tokens || b.rows % b.tokens || b.rows * chunks > kRowThreads ||
                        (cache && b.rows * chunks % 32)) {
                        std::printf("%d tokens, %d heads, %d chunks, %d SMs: %d x %d\n", (int)tokens, heads, chunks, sms, b.tokens, b.rows);
                        return 1;
                    }
                    most = b.tokens > most ? b.tokens : most;
                }
    return most == kBlockTokens ? 0 : 2;
}
""")
    subprocess.run([cxx, "-std=c++17", "-O1", str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, f"exit {r.returncode}: {r.stdout}{r.stderr}"


@pytest.mark.parametrize("d", [64, 128])
def test_a_workspace_serves_every_batch_and_head_count(d):
    # the tickets, then for each of two blocks an SM two pieces of 16 rows of d + 2 floats
    sizes = {ops.wici_paged_attention_workspace_bytes(cache(kv=kv, d=d), kv * group, b)
             for kv in (1, 8) for group in (1, 4, 16, 71) for b in (0, 1, 64, 65535)}
    size, = sizes
    blocks, rest = divmod(size - ops.WICI_ATTN_ZEROED, 2 * 16 * (d + 2) * 4)
    assert rest == 0 and blocks >= 2 and blocks % 2 == 0 and blocks * 4 <= ops.WICI_ATTN_ZEROED
