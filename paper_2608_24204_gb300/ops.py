"""ctypes binding of include/wici_ops.h: rotary positions, a paged key-value cache and
attention over it, for engines that own their device memory.

Every entry point is exposed under its own name (argument marshalling only).  `Rope` and
`PagedKV` take torch tensors: they check shapes, types and devices, and enqueue on torch's
current stream.  There is no fallback: without libwici.so or a GPU these calls raise.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import wici as _w
from .wici import WiciError, _check  # noqa: F401

WICI_BF16, WICI_F16, WICI_F32 = 0, 1, 2
WICI_BAD_SLOT, WICI_BAD_PAGE, WICI_BAD_LENGTH = 1, 2, 4
WICI_ROPE_NONE, WICI_ROPE_LINEAR, WICI_ROPE_BANDS, WICI_ROPE_YARN = 0, 1, 2, 3
WICI_KV_BF16, WICI_KV_INT8, WICI_KV_E4M3, WICI_KV_E2M1 = 0, 1, 2, 4

PAGE_TOKENS = 16
WICI_ATTN_ZEROED = 16384     # bytes at the start of an attention workspace that are zero before its first use
SCALINGS = {"none": WICI_ROPE_NONE, "linear": WICI_ROPE_LINEAR, "bands": WICI_ROPE_BANDS, "yarn": WICI_ROPE_YARN}
FORMATS = {"bf16": WICI_KV_BF16, "int8": WICI_KV_INT8, "e4m3": WICI_KV_E4M3, "e2m1": WICI_KV_E2M1}
_DTYPES = {torch.bfloat16: WICI_BF16, torch.float16: WICI_F16, torch.float32: WICI_F32}

# the entry points declared in include/wici_ops.h
EXPORTS = ("wici_rope_make_plan", "wici_rope", "wici_kv_page_bytes", "wici_kv_append", "wici_kv_read",
           "wici_paged_attention_workspace_bytes", "wici_paged_attention", "wici_selected_attention",
           "wici_kv_bounds_bytes", "wici_kv_bounds_update", "wici_kv_select", "wici_kv_view")


class wici_heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class wici_rope_spec(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_double), ("factor", ctypes.c_double), ("low", ctypes.c_double),
                ("high", ctypes.c_double), ("gain", ctypes.c_double), ("original_len", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("scaling", ctypes.c_int32)]


class wici_rope_plan(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_uint64 * 128), ("gain", ctypes.c_float), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class wici_kv_cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("format", ctypes.c_int32)]


class wici_attn_shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("window", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class wici_kv_bounds(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_stride", ctypes.c_int64)]


class wici_select_shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("keep", ctypes.c_int32),
                ("first", ctypes.c_int32), ("recent", ctypes.c_int32)]


_lib = None
_fast = {}                   # the same entry points taking addresses and packed structures, for `Rope` and `PagedKV`


def lib():
    """libwici.so with the signatures of this header's entry points."""
    global _lib
    if _lib is None:
        L = _w.lib()
        P, i32, i64, vp = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        hp, cp = P(wici_heads), P(wici_kv_cache)
        L.wici_rope_make_plan.argtypes = [P(wici_rope_spec), P(wici_rope_plan)]
        L.wici_rope.argtypes = [vp, P(wici_rope_plan), i32, vp, i64, hp, hp]
        L.wici_kv_page_bytes.argtypes = [i32, i32, i32]
        L.wici_kv_append.argtypes = [vp, cp, vp, i64, hp, hp, P(wici_rope_plan), vp, hp, hp, vp]
        L.wici_kv_read.argtypes = [vp, cp, vp, i64, hp, hp, vp]
        L.wici_paged_attention_workspace_bytes.argtypes = [cp, i32, i32, P(ctypes.c_size_t)]
        L.wici_paged_attention.argtypes = [vp, cp, P(wici_attn_shape), vp, vp, hp, hp, vp, vp, vp]
        L.wici_selected_attention.argtypes = L.wici_paged_attention.argtypes
        L.wici_kv_bounds_bytes.argtypes = [i32, i32]
        L.wici_kv_bounds_update.argtypes = [vp, cp, P(wici_kv_bounds), vp, i64, vp]
        L.wici_kv_select.argtypes = [vp, cp, P(wici_kv_bounds), P(wici_select_shape), vp, vp, hp, vp, vp, vp, vp]
        L.wici_kv_view.argtypes = [vp, i32, cp, P(vp), P(i32)]
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        L.wici_kv_page_bytes.restype = L.wici_kv_bounds_bytes.restype = i64
        for name, types in (("wici_rope", [vp, vp, i32, vp, i64, vp, vp]), ("wici_kv_append", [vp, vp, vp, i64] + [vp] * 7),
                            ("wici_kv_read", [vp, vp, vp, i64, vp, vp, vp]), ("wici_paged_attention", [vp] * 10),
                            ("wici_selected_attention", [vp] * 10), ("wici_kv_bounds_update", [vp, vp, vp, vp, i64, vp]),
                            ("wici_kv_select", [vp] * 11)):
            _fast[name] = L[name]          # a function object of its own
            _fast[name].argtypes, _fast[name].restype = types, ctypes.c_int
        _lib = L
    return _lib


# ---------------------------------------------------------------- thin wrappers
def wici_rope_make_plan(spec: wici_rope_spec) -> wici_rope_plan:
    plan = wici_rope_plan()
    _check(lib().wici_rope_make_plan(spec, plan))
    return plan


def wici_rope(stream: int, plan: wici_rope_plan, inverse: int, positions: int, tokens: int, x: wici_heads,
              y: wici_heads) -> None:
    _check(lib().wici_rope(stream, plan, inverse, positions, tokens, x, y))


def wici_kv_page_bytes(fmt: int, n_kv_heads: int, head_dim: int) -> int:
    return int(lib().wici_kv_page_bytes(fmt, n_kv_heads, head_dim))


def wici_kv_append(stream: int, cache: wici_kv_cache, slots: int, tokens: int, k: wici_heads, v: wici_heads,
                   rope: wici_rope_plan | None = None, positions: int | None = None, q: wici_heads | None = None,
                   q_out: wici_heads | None = None, status: int | None = None) -> None:
    _check(lib().wici_kv_append(stream, cache, slots, tokens, k, v, rope, positions, q, q_out, status))


def wici_kv_read(stream: int, cache: wici_kv_cache, slots: int, tokens: int, k: wici_heads | None,
                 v: wici_heads | None, status: int | None = None) -> None:
    _check(lib().wici_kv_read(stream, cache, slots, tokens, k, v, status))


def wici_paged_attention_workspace_bytes(cache: wici_kv_cache, n_q_heads: int, batch: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().wici_paged_attention_workspace_bytes(cache, n_q_heads, batch, out))
    return int(out.value)


def wici_paged_attention(stream: int, cache: wici_kv_cache, shape: wici_attn_shape, pages: int, lengths: int,
                         q: wici_heads, out: wici_heads, lse: int | None, workspace: int,
                         status: int | None = None) -> None:
    _check(lib().wici_paged_attention(stream, cache, shape, pages, lengths, q, out, lse, workspace, status))


def wici_selected_attention(stream: int, cache: wici_kv_cache, shape: wici_attn_shape, pages: int, lengths: int,
                            q: wici_heads, out: wici_heads, lse: int | None, workspace: int,
                            status: int | None = None) -> None:
    _check(lib().wici_selected_attention(stream, cache, shape, pages, lengths, q, out, lse, workspace, status))


def wici_kv_bounds_bytes(n_kv_heads: int, head_dim: int) -> int:
    return int(lib().wici_kv_bounds_bytes(n_kv_heads, head_dim))


def wici_kv_bounds_update(stream: int, cache: wici_kv_cache, bounds: wici_kv_bounds, last: int, count: int,
                          status: int | None = None) -> None:
    _check(lib().wici_kv_bounds_update(stream, cache, bounds, last, count, status))


def wici_kv_select(stream: int, cache: wici_kv_cache, bounds: wici_kv_bounds, shape: wici_select_shape, pages: int,
                   lengths: int, q: wici_heads, out_pages: int, out_lengths: int, out_blocks: int | None = None,
                   status: int | None = None) -> None:
    _check(lib().wici_kv_select(stream, cache, bounds, shape, pages, lengths, q, out_pages, out_lengths, out_blocks, status))


def wici_kv_view(ctx, layer: int):
    """(cache, device address of the page table, its entries) of a context's layer."""
    cache, pages, n = wici_kv_cache(), ctypes.c_void_p(), ctypes.c_int32()
    _check(lib().wici_kv_view(ctx, layer, cache, pages, n))
    return cache, int(pages.value), int(n.value)


# ------------------------------------------------------------- tensors
_pack_heads = struct.Struct("@Pqqii").pack       # a wici_heads
_pack_shape = struct.Struct("@iiif").pack        # a wici_attn_shape
_pack_select = struct.Struct("@iiiii").pack      # a wici_select_shape
# torch's own short cuts past Stream objects, where this torch has them (2 us of a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _bad_heads(t, head_dim, device, what):
    if t.dim() != 3 or t.shape[2] != head_dim:
        raise ValueError(f"{what}: expected [tokens, heads, {head_dim}], got {tuple(t.shape)}")
    if t.dtype not in _DTYPES:
        raise TypeError(f"{what}: expected bfloat16, float16 or float32, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{what}: on {t.device}, expected cuda:{device}")
    raise ValueError(f"{what}: the elements of a head are not adjacent")


def _heads(t: torch.Tensor, head_dim: int, device: int, what: str):
    """(token stride, head stride, heads, type) of a [tokens][heads][head_dim] tensor on the device."""
    shape, stride, code = t.shape, t.stride(), _DTYPES.get(t.dtype)
    if code is None or len(shape) != 3 or shape[2] != head_dim or t.get_device() != device or stride[2] != 1:
        _bad_heads(t, head_dim, device, what)
    return _pack_heads(t.data_ptr(), stride[0], stride[1], shape[1], code)


def heads_of(t: torch.Tensor, head_dim: int, device: torch.device, what: str) -> wici_heads:
    """A [tokens][heads][head_dim] tensor as the library takes it."""
    return wici_heads.from_buffer_copy(_heads(t, head_dim, -1 if device.type == "cpu" else device.index, what))


def _ints(t: torch.Tensor, shape: tuple, device: int, what: str) -> int:
    if t.dtype != torch.int32 or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what}: expected contiguous int32 {list(shape)} on cuda:{device}, got {t.dtype} "
                         f"{list(t.shape)} on {t.device}")
    return t.data_ptr()


def _stream(device: int) -> int:
    """torch's current stream; the library launches on the current device."""
    if device < 0:
        raise ValueError("expected CUDA tensors")
    if device != _raw_device():
        raise ValueError(f"tensors are on cuda:{device} but the current device is cuda:{_raw_device()}")
    return _raw_stream(device) if _raw_stream else torch.cuda.current_stream(device).cuda_stream


class _Rotation(torch.autograd.Function):
    """A rotation that autograd sees: its gradient is the rotation back, with the same gain."""

    @staticmethod
    def forward(ctx, x, positions, rope, inverse):
        ctx.rope, ctx.inverse = rope, inverse
        ctx.save_for_backward(positions)
        return rope.apply(x, positions, inverse=inverse)

    @staticmethod
    def backward(ctx, dy):
        positions, = ctx.saved_tensors
        return ctx.rope.apply(dy if dy.stride(2) == 1 else dy.contiguous(), positions, inverse=not ctx.inverse), None, None, None


class Rope:
    """Rotary positions of heads of `head_dim`: see wici_rope_spec for the scaling rules."""

    def __init__(self, head_dim: int, theta: float, rot_dim: int | None = None, interleaved: bool = False,
                 scaling: str = "none", factor: float = 1.0, original_len: int = 0, low: float = 0.0,
                 high: float = 0.0, gain: float = 0.0):
        if scaling not in SCALINGS:
            raise ValueError(f"scaling {scaling!r}: expected one of {', '.join(SCALINGS)}")
        self.head_dim = head_dim
        self.plan = wici_rope_make_plan(wici_rope_spec(
            theta, factor, low, high, gain, original_len, head_dim, head_dim if rot_dim is None else rot_dim,
            int(interleaved), SCALINGS[scaling]))
        self._plan = ctypes.addressof(self.plan)

    def apply(self, x: torch.Tensor, positions: torch.Tensor, out: torch.Tensor | None = None,
              inverse: bool = False) -> torch.Tensor:
        """x [tokens, heads, head_dim] rotated by `positions` (int32 [tokens]); with `inverse` the gradient of
        that with respect to x, from the gradient of its result.  `out` may be x.  Autograd sees the call where `out`
        is not given."""
        if out is None and x.requires_grad and torch.is_grad_enabled():
            return _Rotation.apply(x, positions, self, inverse)
        device, d = x.get_device(), self.head_dim
        stream = _stream(device)
        hx = _heads(x, d, device, "x")
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        elif out.shape != x.shape:
            raise ValueError(f"out: expected {list(x.shape)}, got {list(out.shape)}")
        n = x.shape[0]
        _check(_fast["wici_rope"](stream, self._plan, 1 if inverse else 0, _ints(positions, (n,), device, "positions"), n,
                                  hx, _heads(out, d, device, "out")))
        return out


class PagedKV:
    """A paged key-value cache of one layer: `n_pages` pages of 16 tokens in a torch buffer (or in `data`, a uint8
    tensor of whole pages).  Slot s is place s % 16 of page s // 16.

    A buffer made here and the word that `check` reads are cleared on the stream that is current here: calls on another
    stream come after that, as with any tensor.  Autograd does not see the calls."""

    def __init__(self, n_kv_heads: int, head_dim: int, fmt: str = "bf16", n_pages: int | None = None,
                 data: torch.Tensor | None = None, device=None):
        if fmt not in FORMATS:
            raise ValueError(f"format {fmt!r}: expected one of {', '.join(FORMATS)}")
        self.n_kv_heads, self.head_dim, self.fmt = n_kv_heads, head_dim, fmt
        page = wici_kv_page_bytes(FORMATS[fmt], n_kv_heads, head_dim)
        if page == 0:
            raise ValueError(f"{n_kv_heads} heads of {head_dim}: head_dim must be 64 or 128")
        if data is None:
            if n_pages is None:
                raise ValueError("n_pages or data is needed")
            data = torch.zeros(n_pages * page, dtype=torch.uint8, device=device or "cuda")
        if data.dtype != torch.uint8 or not data.is_contiguous() or data.numel() % page:
            raise ValueError(f"data: expected contiguous uint8 in whole pages of {page} bytes")
        self.data, self.device, self._device = data, data.device, data.get_device()
        self.n_pages = data.numel() // page
        self.cache = wici_kv_cache(data.data_ptr(), page, self.n_pages, n_kv_heads, head_dim, FORMATS[fmt])
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._cache, self._status = ctypes.addressof(self.cache), self.status.data_ptr()
        self._workspaces, self._served = {}, {}   # per stream; the largest batch that its workspace is known to take, per heads
        if self._device >= 0 and self._device == torch.cuda.current_device():
            self.workspace_bytes(n_kv_heads, 1)   # sets the attention kernels up, before a capture may need them

    def append(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, rope: Rope | None = None,
               positions: torch.Tensor | None = None, q: torch.Tensor | None = None,
               q_out: torch.Tensor | None = None) -> torch.Tensor | None:
        """Write k, v [tokens, n_kv_heads, head_dim] at `slots` (int32 [tokens], distinct; negative: skipped).
        With a rope, k is rotated by `positions` on the way, and q into q_out, which is returned (a new tensor
        unless given; it may be q)."""
        dev, d = self._device, self.head_dim
        stream = _stream(dev)
        n = k.shape[0]
        if v.shape[0] != n:
            raise ValueError(f"v: expected {n} tokens, got {v.shape[0]}")
        hq = ho = None
        if q is not None:
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
            if q.shape[0] != n or q_out.shape != q.shape:
                raise ValueError(f"q, q_out: expected {n} tokens and one shape, got {list(q.shape)}, {list(q_out.shape)}")
            hq, ho = _heads(q, d, dev, "q"), _heads(q_out, d, dev, "q_out")
        elif q_out is not None:
            raise ValueError("q_out without q")
        _check(_fast["wici_kv_append"](
            stream, self._cache, _ints(slots, (n,), dev, "slots"), n, _heads(k, d, dev, "k"), _heads(v, d, dev, "v"),
            None if rope is None else rope._plan, None if positions is None else _ints(positions, (n,), dev, "positions"),
            hq, ho, self._status))
        return q_out

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, out=None):
        """(k, v) [slots, n_kv_heads, head_dim] at `slots` (int32; negative: zeros), into `out` when given."""
        dev, d = self._device, self.head_dim
        stream = _stream(dev)
        n = slots.shape[0]
        if out is None:
            out = tuple(torch.empty((n, self.n_kv_heads, d), dtype=dtype, device=self.device) for _ in range(2))
        k, v = out
        if k.shape[0] != n or v.shape[0] != n:
            raise ValueError(f"out: expected {n} tokens, got {k.shape[0]} and {v.shape[0]}")
        _check(_fast["wici_kv_read"](stream, self._cache, _ints(slots, (n,), dev, "slots"), n, _heads(k, d, dev, "k"),
                                     _heads(v, d, dev, "v"), self._status))
        return k, v

    def attend(self, q: torch.Tensor, pages: torch.Tensor, lengths: torch.Tensor, scale: float | None = None,
               window: int = 0, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
        """One token's attention per sequence: q [batch, heads, head_dim] over the first lengths[b] tokens (the last
        `window` of them, 0: all) of the pages pages[b] (int32 [batch, max_pages], or [batch, n_kv_heads, max_pages]
        where every KV head has pages of its own, as KeyBounds.select gives them; without a window).  scale: head_dim ** -0.5 unless
        given.  Fills lse (float32 [batch, heads]) when given.  The workspace, unless given (`workspace()`), is one
        per stream, or in a graph capture one of that call's own."""
        dev, d = self._device, self.head_dim
        stream = _stream(dev)
        hq = _heads(q, d, dev, "q")
        batch, heads, _ = q.shape
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
        elif out.shape[0] < batch:
            raise ValueError(f"out: {out.shape[0]} rows for a batch of {batch}")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != (batch, heads) or not lse.is_contiguous() or
                                lse.get_device() != dev):
            raise ValueError(f"lse: expected contiguous float32 {[batch, heads]} on cuda:{dev}")
        selected = pages.dim() == 3
        if not selected and pages.dim() != 2:
            raise ValueError("pages: expected [batch, max_pages] or [batch, n_kv_heads, max_pages]")
        if workspace is None:
            workspace = self._workspace_for(stream, heads, batch)
        elif workspace.get_device() != dev or not workspace.is_contiguous() or \
                workspace.numel() * workspace.element_size() < self.workspace_bytes(heads, batch):
            raise ValueError(f"workspace: expected {self.workspace_bytes(heads, batch)} bytes on cuda:{dev}")
        columns = pages.shape[-1]
        shape = _pack_shape(batch, columns, window, d ** -0.5 if scale is None else scale)
        table = _ints(pages, (batch, self.n_kv_heads, columns) if selected else (batch, columns), dev, "pages")
        _check(_fast["wici_selected_attention" if selected else "wici_paged_attention"](
            stream, self._cache, shape, table, _ints(lengths, (batch,), dev, "lengths"),
            hq, _heads(out, d, dev, "out"), None if lse is None else lse.data_ptr(), workspace.data_ptr(), self._status))
        return out

    def workspace_bytes(self, n_q_heads: int, batch: int) -> int:
        return wici_paged_attention_workspace_bytes(self.cache, n_q_heads, batch)

    def workspace(self, n_q_heads: int, batch: int) -> torch.Tensor:
        """A workspace of attend's, for calls that are ordered with each other."""
        ws = torch.empty(self.workspace_bytes(n_q_heads, batch), dtype=torch.uint8, device=self.device)
        ws[:WICI_ATTN_ZEROED].zero_()
        return ws

    def _workspace_for(self, stream: int, n_q_heads: int, batch: int) -> torch.Tensor:
        if torch.cuda.is_current_stream_capturing():
            return self.workspace(n_q_heads, batch)   # zeroed by every replay, in the graph's own memory
        if self._served.get((stream, n_q_heads), -1) < batch:
            kept = self._workspaces.get(stream)
            if kept is None or kept.numel() < self.workspace_bytes(n_q_heads, batch):
                self._workspaces[stream] = self.workspace(n_q_heads, batch)
            self._served[stream, n_q_heads] = batch
        return self._workspaces[stream]

    def check(self) -> None:
        """Waits for the current stream and raises if a call on it (a KeyBounds' among them) met a slot, page or length outside the cache
        (which clears the record)."""
        bits = int(self.status.item())
        if bits:
            self.status.zero_()
            what = [n for b, n in ((WICI_BAD_SLOT, "a slot"), (WICI_BAD_PAGE, "a page"), (WICI_BAD_LENGTH, "a length"))
                    if bits & b]
            raise WiciError(_w.WICI_E_ARG, f"paged cache: {' and '.join(what)} outside the cache or page table")


class KeyBounds:
    """Bounds of the keys in each page of a cache, by which `select` chooses the pages that a step attends to: the largest
    and the smallest key element by element as int8 `codes` [page, kv head, 2, head_dim] under `scales` [page, kv head],
    in a torch buffer (or in `data`, a uint8 tensor of a record for each page).

    A step of a long context: PagedKV.append, `update` with its slots, `select`, PagedKV.attend over what that gives.
    The cache's `check` reports slots, pages and lengths outside it.  Autograd does not see the calls."""

    def __init__(self, cache: PagedKV, data: torch.Tensor | None = None):
        kv, d = cache.n_kv_heads, cache.head_dim
        record = wici_kv_bounds_bytes(kv, d)
        if data is None:
            data = torch.zeros(cache.n_pages * record, dtype=torch.uint8, device=cache.device)
        if data.dtype != torch.uint8 or not data.is_contiguous() or data.numel() != cache.n_pages * record or data.device != cache.device:
            raise ValueError(f"data: expected contiguous uint8 [{cache.n_pages * record}] on {cache.device}: records of {record} bytes")
        self.cache, self.data = cache, data
        rows = data.view(cache.n_pages, record)
        self.codes = rows[:, :kv * 2 * d].view(torch.int8).unflatten(1, (kv, 2, d))
        self.scales = rows[:, kv * 2 * d:kv * (2 * d + 4)].view(torch.float32)
        self.bounds = wici_kv_bounds(data.data_ptr(), record)
        self._bounds = ctypes.addressof(self.bounds)

    def update(self, last: torch.Tensor) -> None:
        """Bounds of the pages of slots `last` (int32 [n]; each the last token of its page, a page at most once; negative:
        skipped), over a page's places up to that slot."""
        c = self.cache
        stream = _stream(c._device)
        n = last.shape[0]
        _check(_fast["wici_kv_bounds_update"](stream, c._cache, self._bounds, _ints(last, (n,), c._device, "last"), n, c._status))

    def select(self, q: torch.Tensor, pages: torch.Tensor, lengths: torch.Tensor, keep: int, first: int = 1, recent: int = 1,
               out: tuple[torch.Tensor, torch.Tensor] | None = None, blocks: torch.Tensor | None = None):
        """(pages int32 [batch, n_kv_heads, keep], lengths int32 [batch]) for PagedKV.attend: of the pages pages[b] (int32
        [batch, max_pages]) of a sequence of lengths[b] tokens the first `first`, the last `recent` and those that score
        highest against q [batch, heads, head_dim], `keep` in all, for each KV head.  Into `out` when given; fills `blocks`
        (as the pages) with their columns in `pages` when given."""
        c = self.cache
        dev, kv = c._device, c.n_kv_heads
        stream = _stream(dev)
        hq = _heads(q, c.head_dim, dev, "q")
        batch = q.shape[0]
        if pages.dim() != 2:
            raise ValueError("pages: expected [batch, max_pages]")
        if keep < 1:
            raise ValueError(f"keep: expected at least 1, got {keep}")
        if out is None:
            out = (torch.empty((batch, kv, keep), dtype=torch.int32, device=c.device), torch.empty(batch, dtype=torch.int32, device=c.device))
        chosen, held = out
        shape = _pack_select(batch, pages.shape[1], keep, first, recent)
        _check(_fast["wici_kv_select"](
            stream, c._cache, self._bounds, shape, _ints(pages, (batch, pages.shape[1]), dev, "pages"),
            _ints(lengths, (batch,), dev, "lengths"), hq, _ints(chosen, (batch, kv, keep), dev, "out pages"),
            _ints(held, (batch,), dev, "out lengths"), None if blocks is None else _ints(blocks, (batch, kv, keep), dev, "blocks"),
            c._status))
        return chosen, held
