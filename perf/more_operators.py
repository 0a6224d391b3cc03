"""Operators of long contexts whose speed is measured: a paged key-value cache held in 4 bits
with the attention that reads it, and attention of one new token per sequence over the blocks
of a cache that a cheap score selects.

The cache is a byte buffer of pages.  A page holds 16 tokens: [K|V][kv head] blocks.
* e2m1: [16][head_dim / 2] bytes of two codes each (the lower half first), then [16][head_dim / 16]
  e4m3 scales of 16 elements each, then 16 fp32 scales, one per token:
  value = code * block scale * scale, with scale = max |x| of the token's head / 2688,
  block scale = (max |x| of the 16) / (6 scale) as e4m3, code = x / (block scale * scale) as e2m1.
* bf16, and e4m3 or int8 codes followed by 16 fp32 scales.
A slot is page * 16 + place.

Bounds are a byte buffer beside it, one record per page: [kv head][largest|smallest][head_dim] int8
codes of the page's keys, element by element, then one fp32 scale per kv head (records are padded
to 16 bytes).  A query meets a page's bounds in whole numbers: q as whole numbers up to 1023, the
larger end of each element's range where q is positive and the smaller one where it is negative.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TOP = {"int8": 127.0, "e4m3": 448.0, "e2m1": 2688.0}      # the largest value that stands beside a scale
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LEVELS = 1023.0                                           # of a query's whole numbers


def _case(name, kind, **dims):
    return dict({"name": name, "kind": kind}, **dims)


def listed():
    return [
        # two chats of a few hundred tokens take their next step: launch and latency
        _case("step e2m1 short", "attention", batch=2, shortest=100, longest=300, q_heads=32, kv_heads=8, dim=128,
              dtype="bf16", format="e2m1", window=0, step=True),
        # many clients of the 14B shape (five query heads to a KV head) take a step
        _case("step e2m1 batch", "attention", batch=64, shortest=1000, longest=8192, q_heads=40, kv_heads=8, dim=128,
              dtype="bf16", format="e2m1", window=0, step=True),
        # two documents in a long context of the 8B shape: the split over the length
        _case("attention e2m1 long", "attention", batch=2, shortest=100001, longest=131072, q_heads=32, kv_heads=8, dim=128,
              dtype="bf16", format="e2m1", window=0, step=False),
        # the 1B shape in fp32 with a sliding window
        _case("attention e2m1 window", "attention", batch=48, shortest=300, longest=16000, q_heads=32, kv_heads=8, dim=64,
              dtype="f32", format="e2m1", window=4096, step=False),
        # prompts of several clients written at once, and read back as the next turn's dense prefill does
        _case("prompts and back", "append", tokens=16384, run=2731, kv_heads=8, dim=128, dtype="bf16", format="e2m1", read="bf16"),
        # keys and values of an fp32 engine, a ragged count of tokens
        _case("f32 and back", "append", tokens=1251, run=417, kv_heads=8, dim=64, dtype="f32", format="e2m1", read="f32"),
        # a cached prefix of many pages read back
        _case("read prefix e2m1", "read", tokens=30011, kv_heads=8, dim=128, dtype="bf16", format="e2m1"),
        # the page that each client's new token stands in gets its bounds again
        _case("bounds step", "bounds", pages=64, full=False, kv_heads=8, dim=128, format="bf16"),
        # every page of long prompts that were just written
        _case("bounds prompts", "bounds", pages=4096, full=True, kv_heads=8, dim=128, format="e4m3"),
        # one agent's context of the 8B shape, a kilotoken of it read a step
        _case("sparse short", "sparse", batch=1, shortest=8448, longest=8448, q_heads=32, kv_heads=8, dim=128, dtype="bf16",
              format="bf16", keep=64, first=1, recent=2),
        # clients of the 8B shape at long and ragged contexts
        _case("sparse batch", "sparse", batch=32, shortest=2000, longest=32768, q_heads=32, kv_heads=8, dim=128, dtype="bf16",
              format="bf16", keep=128, first=1, recent=4),
        # documents of a long context over a cache in 4 bits
        _case("sparse long e2m1", "sparse", batch=4, shortest=100001, longest=131072, q_heads=32, kv_heads=8, dim=128,
              dtype="bf16", format="e2m1", keep=256, first=2, recent=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "append", "read", "bounds", "sparse", "sparse", "sparse"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    dim = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8])
    if kind == "append":
        tokens = _log(rng, 1, 16384)
        return _unnamed(kind, tokens=tokens, run=rng.randint(1, tokens), kv_heads=kv, dim=dim, dtype=dtype, format="e2m1",
                        read=rng.choice(["bf16", "f16", "f32"]) if tokens < 8192 else "bf16")
    if kind == "read":
        return _unnamed(kind, tokens=_log(rng, 1, 30000), kv_heads=kv, dim=dim, dtype=dtype, format="e2m1")
    if kind == "bounds":
        return _unnamed(kind, pages=_log(rng, 1, 4096), full=rng.random() < 0.5, kv_heads=kv, dim=dim,
                        format=rng.choice(["bf16", "int8", "e4m3", "e2m1"]))
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    if kind == "attention":
        batch = _log(rng, 1, 96)
        longest = _log(rng, 1, min(131072, 200000 // batch))
        shortest = _log(rng, 1, longest)
        return _unnamed(kind, batch=batch, shortest=shortest, longest=longest, q_heads=kv * group, kv_heads=kv, dim=dim, dtype=dtype,
                        format="e2m1", window=rng.choice([0, 0, 0, rng.randint(1, 5000)]), step=shortest > 64 and rng.random() < 0.7)
    batch = _log(rng, 1, 96)
    longest = _log(rng, 1, min(131072, 400000 // batch))
    first, recent = rng.randint(0, 4), rng.randint(1, 8)
    return _unnamed(kind, batch=batch, shortest=_log(rng, 1, longest), longest=longest, q_heads=kv * group, kv_heads=kv, dim=dim,
                    dtype=dtype, format=rng.choice(["bf16", "int8", "e4m3", "e2m1"]), keep=_log(rng, first + recent, 256),
                    first=first, recent=recent)


def _unnamed(kind, **dims):
    return dict({"kind": kind}, **dims)


# ------------------------------------------------------------------ inputs --
def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(g, *shape):
    """Keys as projections give them: a few channels far larger than the others, the same in every token."""
    gain = torch.exp(0.6 * _normal(g, *shape[-2:]))
    return _normal(g, *shape).mul_(gain).add_(0.5 * gain)


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)


def _block(dim, fmt):
    """Bytes of one [K or V][kv head] block of a page."""
    return PAGE * {"bf16": 2 * dim, "int8": dim + 4, "e4m3": dim + 4, "e2m1": dim // 2 + dim // 16 + 4}[fmt]


def _parts(pool, kv_heads, dim, fmt):
    """Views of a pool: the values or codes [page][K|V][head][16][..], e2m1's block scales and the tokens' scales (None where
    a format has none)."""
    if fmt == "bf16":
        return pool.view(torch.bfloat16).view(-1, 2, kv_heads, PAGE, dim), None, None
    blocks = pool.view(-1, 2, kv_heads, _block(dim, fmt))
    scales = blocks.view(torch.float32)[..., -PAGE:]
    if fmt == "e2m1":
        half, each = dim // 2, dim // 16
        return (blocks[..., :PAGE * half].unflatten(-1, (PAGE, half)),
                blocks[..., PAGE * half:PAGE * (half + each)].unflatten(-1, (PAGE, each)), scales)
    return blocks[..., :PAGE * dim].unflatten(-1, (PAGE, dim)), None, scales


def _quantised(x, fmt):
    """(codes as stored, block scales, scales) of rows x [..][dim]; e2m1's in x's own precision: quotients lie next to borders."""
    scale = (x.abs().amax(-1) / TOP[fmt]).float()
    if fmt != "e2m1":
        y = x / scale.clamp_min(1e-37).unsqueeze(-1)
        return (y.round().to(torch.int8) if fmt == "int8" else y.clamp(-448, 448).to(torch.float8_e4m3fn)).view(torch.uint8), None, scale
    x = x.unflatten(-1, (-1, 16))
    wide = scale.to(x.dtype).unsqueeze(-1)
    grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).to(x.dtype)   # by code
    each = _nearest(x.abs().amax(-1) / (6.0 * wide).clamp_min(1e-37), grid)
    y = x.abs() / (grid[each] * wide).clamp_min(1e-37).unsqueeze(-1)
    code = (_nearest(y, torch.tensor(E2M1, dtype=x.dtype, device="cuda")) + 8 * (x < 0).int()).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, each.to(torch.uint8), scale


def _nearest(y, grid):
    """The place of the nearest number of a grid, the even one of two that are as near."""
    middle = (grid[1:] + grid[:-1]) / 2
    at = torch.bucketize(y, middle, out_int32=True)
    return at + ((at & 1) * (y == middle[at.clamp_max(len(middle) - 1)])).int()


def _values_of(codes, each, scales, fmt, to=torch.float32):
    """What codes as stored stand for."""
    if fmt == "bf16":
        return codes.to(to)
    if fmt != "e2m1":
        return codes.contiguous().view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).to(to) * scales.to(to).unsqueeze(-1)
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=to, device="cuda")
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)
    each = each.contiguous().view(torch.float8_e4m3fn).to(to)
    return ((v.unflatten(-1, (-1, 16)) * each.unsqueeze(-1)).flatten(-2)) * scales.to(to).unsqueeze(-1)


def _store(pool, page, which, place, x, case):
    values, each, scales = _parts(pool, case["kv_heads"], case["dim"], case["format"])
    if case["format"] == "bf16":
        values[page, which, :, place] = x.to(torch.bfloat16)
        return
    c, e, s = _quantised(x.double() if case["format"] == "e2m1" else x, case["format"])
    values[page, which, :, place] = c
    scales[page, which, :, place] = s
    if e is not None:
        each[page, which, :, place] = e


def _filled(g, pages, case, topic=0.0):
    """A pool as earlier calls left it: every slot holds a token.  topic: how much a page's keys have in common."""
    kv, dim, fmt = case["kv_heads"], case["dim"], case["format"]
    pool = torch.zeros(pages * 2 * kv * _block(dim, fmt), dtype=torch.uint8, device="cuda")
    values, each, scales = _parts(pool, kv, dim, fmt)
    step = max(1, (1 << 25) // (2 * kv * PAGE * dim))
    gain = torch.exp(0.6 * _normal(g, 2, kv, 1, dim))
    gain[1] = 1.0
    for a in range(0, pages, step):
        n = min(step, pages - a)
        x = _normal(g, n, 2, kv, PAGE, dim)
        if topic:
            x[:, 0] += topic * _normal(g, n, kv, 1, dim)
        x = x.mul_(gain)
        if fmt == "bf16":
            values[a:a + n] = x.to(torch.bfloat16)
            continue
        c, e, s = _quantised(x, fmt)
        values[a:a + n] = c
        scales[a:a + n] = s
        if e is not None:
            each[a:a + n] = e
    return pool


def _record(kv_heads, dim):
    return (kv_heads * (2 * dim + 4) + 15) // 16 * 16


def _bounds_parts(bounds, kv_heads, dim):
    """Views of bounds: codes [page][head][largest|smallest][dim], scales [page][head]."""
    rows = bounds.view(-1, _record(kv_heads, dim))
    n = kv_heads * 2 * dim
    return rows[:, :n].view(torch.int8).unflatten(-1, (kv_heads, 2, dim)), rows[:, n:n + 4 * kv_heads].view(torch.float32)


def _bound(pool, bounds, page, fill, case):
    """The bounds of pages whose first `fill` places hold tokens."""
    values, each, scales = _parts(pool, case["kv_heads"], case["dim"], case["format"])
    k = _values_of(values[page, 0], None if each is None else each[page, 0], None if scales is None else scales[page, 0], case["format"])
    there = (torch.arange(PAGE, device="cuda") < fill.unsqueeze(1))[:, None, :, None]
    hi = torch.where(there, k, torch.tensor(-math.inf, device="cuda")).amax(2)
    lo = torch.where(there, k, torch.tensor(math.inf, device="cuda")).amin(2)
    scale = torch.maximum(hi.abs(), lo.abs()).amax(-1) / 127.0
    codes = (torch.stack((hi, lo), 2) / scale.clamp_min(1e-37)[..., None, None]).round().to(torch.int8)
    at, to = _bounds_parts(bounds, case["kv_heads"], case["dim"])
    at[page] = codes
    to[page] = scale


def _tables(g, lengths, longest, extra=3):
    """A page table in any order, -1 past a sequence's end, and the number of pages."""
    most = -(-longest // PAGE)
    need = (lengths.long() + PAGE - 1) // PAGE
    total = int(need.sum()) + extra
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(most, device="cuda")
    flat = (torch.cumsum(need, 0) - need).unsqueeze(1) + at
    return torch.where(at < need.unsqueeze(1), order[flat.clamp_max(total - 1)], -1), total


def prepare(case, seed):
    g = _generator(seed, 29)
    kind, kv, d = case["kind"], case["kv_heads"], case["dim"]
    if kind in ("attention", "sparse"):
        B, nq = case["batch"], case["q_heads"]
        lengths = _ints(g, case["shortest"], case["longest"], B)
        if B > 8 and not case.get("step"):
            lengths[0], lengths[1], lengths[2] = 0, 1, case["longest"]          # a padding row and a first token
        pages, total = _tables(g, lengths, case["longest"])
        s = {"case": case, "pool": _filled(g, total, case, 0.7 if kind == "sparse" else 0.0), "pages": pages, "lengths": lengths,
             "scale": d ** -0.5, "q": (2.0 * _normal(g, B, nq, d)).to(TORCH[case["dtype"]]),
             "out": torch.zeros((B, nq, d), dtype=TORCH[case["dtype"]], device="cuda"), "lse": torch.zeros((B, nq), device="cuda")}
        if kind == "sparse":
            s["bounds"] = torch.zeros(total * _record(kv, d), dtype=torch.uint8, device="cuda")
            step = max(1, (1 << 26) // (kv * PAGE * d))
            fill = torch.full((total,), PAGE, device="cuda")
            some = lengths > 0
            last = lengths[some].long() - 1
            fill[pages[some].gather(1, (last // PAGE).unsqueeze(1)).squeeze(1).long()] = last % PAGE + 1
            for a in range(0, total, step):
                page = torch.arange(a, min(a + step, total), device="cuda")
                _bound(s["pool"], s["bounds"], page, fill[page], case)
            s["selected"] = torch.zeros((B, kv, case["keep"]), dtype=torch.int32, device="cuda")
            s["blocks"] = torch.zeros_like(s["selected"])
            s["held"] = torch.zeros_like(lengths)
        if case.get("step"):
            rows = _keys(g, B, nq + 2 * kv, d).to(TORCH[case["dtype"]])          # the packed q|k|v rows of a projection
            last = lengths.long() - 1
            s |= {"q": rows[:, :nq], "k": rows[:, nq:nq + kv], "v": rows[:, nq + kv:], "positions": lengths - 1,
                  "slots": (pages.gather(1, (last // PAGE).unsqueeze(1)).squeeze(1) * PAGE + last % PAGE).to(torch.int32),
                  "q_out": torch.zeros((B, nq, d), dtype=rows.dtype, device="cuda")}
        return s
    if kind == "bounds":
        n = case["pages"]
        total = n + 2
        order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)[:n]
        fill = torch.full((n,), PAGE, dtype=torch.int32, device="cuda") if case["full"] else _ints(g, 1, PAGE, n)
        return {"case": case, "pool": _filled(g, total, case, 0.7), "last": order * PAGE + fill - 1,
                "bounds": torch.zeros(total * _record(kv, d), dtype=torch.uint8, device="cuda")}
    T = case["tokens"]
    if kind == "read":
        pages = -(-T // PAGE) + 2
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        at = torch.arange(T, device="cuda")
        return {"case": case, "pool": _filled(g, pages, case), "slots": order[at // PAGE] * PAGE + (at % PAGE).to(torch.int32),
                "back": [torch.zeros((T, kv, d), dtype=TORCH[case["dtype"]], device="cuda") for _ in range(2)]}
    # tokens of several sequences, `run` of each: every run starts on a page of its own
    run_ = case["run"]
    runs, per = -(-T // run_), -(-run_ // PAGE)
    order = torch.randperm(runs * per, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(T, device="cuda")
    seq, off = at // run_, at % run_
    rows = _keys(g, T, 2 * kv, d).to(TORCH[case["dtype"]])                      # the k|v part of a projection's rows
    return {"case": case, "slots": order[seq * per + off // PAGE] * PAGE + (off % PAGE).to(torch.int32), "k": rows[:, :kv],
            "v": rows[:, kv:], "pool": torch.zeros(runs * per * 2 * kv * _block(d, case["format"]), dtype=torch.uint8, device="cuda"),
            "back": [torch.zeros((T, kv, d), dtype=TORCH[case["read"]], device="cuda") for _ in range(2)]}


# --------------------------------------------------------------------- run --
def run(s):
    return _RUN[s["case"]["kind"]][1 if own else 0](s)


THETA = 5e5


def _turned(x, positions):
    """x [tokens][heads][dim] with its halves rotated by the positions, in 64 bits: far angles, codes next to a border."""
    half = x.shape[-1] // 2
    f = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    a = (positions.double().unsqueeze(1) * f).unsqueeze(1)
    c, n = torch.cos(a), torch.sin(a)
    u, v = x[..., :half].double(), x[..., half:].double()
    return torch.cat((u * c - v * n, u * n + v * c), -1)


def _write_plain(pool, which, x, slots, case):
    slots = slots.long()
    _store(pool, slots // PAGE, which, slots % PAGE, x, case)


def _read_plain_both(s):
    case = s["case"]
    values, each, scales = _parts(s["pool"], case["kv_heads"], case["dim"], case["format"])
    page, place = s["slots"].long() // PAGE, s["slots"].long() % PAGE
    for which in (0, 1):
        s["back"][which].copy_(_values_of(values[page, which, :, place], each[page, which, :, place], scales[page, which, :, place],
                                          case["format"]))
    return {"k": s["back"][0], "v": s["back"][1]}


def _append_plain(s):
    _write_plain(s["pool"], 0, s["k"].float(), s["slots"], s["case"])
    _write_plain(s["pool"], 1, s["v"].float(), s["slots"], s["case"])
    return _read_plain_both(s)


def _attend_plain(s, q, pages, valid):
    """q [batch][heads][dim] over the tokens of pages [batch][1 or kv heads][..] where valid [batch][tokens]."""
    case = s["case"]
    B, nq, kv, d = case["batch"], case["q_heads"], case["kv_heads"], case["dim"]
    values, each, scales = _parts(s["pool"], kv, d, case["format"])
    pages = pages.long().expand(B, kv, -1).transpose(1, 2)
    head = torch.arange(kv, device="cuda")

    def dense(which):                                                       # [batch][head][key][dim]
        at = (pages, which, head)
        x = _values_of(values[at], None if each is None else each[at], None if scales is None else scales[at], case["format"])
        return x.transpose(1, 2).reshape(B, kv, -1, d)

    k = dense(0)
    x = (q.float().view(B, kv, nq // kv, d) @ k.transpose(2, 3)) * s["scale"]
    del k
    x = x.masked_fill(~valid[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    v = torch.where(valid[:, None, :, None], dense(1), torch.zeros((), device="cuda"))
    o = (p @ v) / torch.where(total == 0, torch.ones_like(total), total)
    s["out"].copy_(o.reshape(B, nq, d))
    s["lse"].copy_((top + torch.log(total)).reshape(B, nq))
    return {"out": s["out"], "lse": s["lse"]}


def _attention_plain(s):
    case, q = s["case"], s["q"]
    if case["step"]:
        q = s["q_out"].copy_(_turned(q, s["positions"]))
        _write_plain(s["pool"], 0, _turned(s["k"], s["positions"]), s["slots"], case)
        _write_plain(s["pool"], 1, s["v"].float(), s["slots"], case)
    at = torch.arange(s["pages"].shape[1] * PAGE, device="cuda")
    n = s["lengths"].unsqueeze(1)
    valid = at < n
    if case["window"]:
        valid &= at >= n - case["window"]
    out = _attend_plain(s, q, s["pages"].unsqueeze(1), valid)
    return dict(out, q=q) if case["step"] else out


def _bounds_plain(s):
    case = s["case"]
    last = s["last"].long()
    _bound(s["pool"], s["bounds"], last // PAGE, last % PAGE + 1, case)
    codes, scales = _bounds_parts(s["bounds"], case["kv_heads"], case["dim"])
    return {"codes": codes, "scales": scales}


def _sparse_plain(s):
    case, pages = s["case"], s["pages"].long()
    B, nq, kv, d, keep = case["batch"], case["q_heads"], case["kv_heads"], case["dim"], case["keep"]
    codes, scales = _bounds_parts(s["bounds"], kv, d)
    q = s["q"].float().view(B, kv, nq // kv, d)
    most = q.abs().amax(-1, keepdim=True)
    whole = (q * (LEVELS / most)).round()
    ends = torch.cat((whole.clamp_min(0.0), whole.clamp_max(0.0)), -1).double()
    dots = ends @ codes[pages].permute(0, 2, 3, 4, 1).reshape(B, kv, 2 * d, -1).double()   # whole numbers below 2^24
    score = (dots.float() * most).amax(2) * scales[pages].transpose(1, 2)                  # [batch][head][page]
    at = torch.arange(pages.shape[1], device="cuda")
    count = ((s["lengths"].long() + PAGE - 1) // PAGE)[:, None, None]
    key = score.double()
    key = torch.where((at < case["first"]) | (at >= count - case["recent"]), torch.tensor(math.inf, dtype=torch.float64, device="cuda"), key)
    key = torch.where(at < count, key, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
    chosen = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    chosen = torch.sort(torch.where(chosen < count, chosen, pages.shape[1]), dim=-1).values   # ascending, those past the end last
    there = chosen < pages.shape[1]
    s["blocks"].fill_(-1)
    s["selected"].fill_(-1)
    s["blocks"][..., :chosen.shape[-1]] = torch.where(there, chosen, -1).int()
    of = pages.gather(1, chosen.clamp_max(pages.shape[1] - 1).flatten(1)).view_as(chosen)
    s["selected"][..., :chosen.shape[-1]] = torch.where(there, of, -1).int()
    n = s["lengths"]
    s["held"].copy_(torch.where(count.flatten() <= keep, n, (keep - 1) * PAGE + (n - 1) % PAGE + 1))
    valid = torch.arange(keep * PAGE, device="cuda") < s["held"].unsqueeze(1)
    out = _attend_plain(s, s["q"], s["selected"], valid)
    return dict(out, blocks=s["blocks"], selected=s["selected"], held=s["held"])


# ---- the framework's operators ----
_ops = None


def _kept(s, name, make):
    """The rope, cache or bounds handle that a program makes once for its shapes."""
    global _ops
    if _ops is None:
        from paper_2608_24204_gb300 import ops
        _ops = ops
    if name not in s:
        s[name] = make()
    return s[name]


def _cache_of(s):
    case = s["case"]
    return _kept(s, "cache", lambda: _ops.PagedKV(case["kv_heads"], case["dim"], case["format"], data=s["pool"]))


def _bounds_of(s):
    cache = _cache_of(s)
    return _kept(s, "key bounds", lambda: _ops.KeyBounds(cache, data=s["bounds"]))


def _read_own(s):
    _cache_of(s).read(s["slots"], out=s["back"])
    return {"k": s["back"][0], "v": s["back"][1]}


def _append_own(s):
    _cache_of(s).append(s["k"], s["v"], s["slots"])
    return _read_own(s)


def _attention_own(s):
    case, cache, q = s["case"], _cache_of(s), s["q"]
    if case["step"]:
        rope = _kept(s, "rope", lambda: _ops.Rope(case["dim"], THETA))
        q = cache.append(s["k"], s["v"], s["slots"], rope=rope, positions=s["positions"], q=q, q_out=s["q_out"])
    cache.attend(q, s["pages"], s["lengths"], scale=s["scale"], window=case["window"], out=s["out"], lse=s["lse"])
    out = {"out": s["out"], "lse": s["lse"]}
    return dict(out, q=q) if case["step"] else out


def _bounds_own(s):
    case = s["case"]
    bounds = _bounds_of(s)
    bounds.update(s["last"])
    return {"codes": bounds.codes, "scales": bounds.scales}


def _sparse_own(s):
    case = s["case"]
    bounds = _bounds_of(s)
    bounds.select(s["q"], s["pages"], s["lengths"], case["keep"], first=case["first"], recent=case["recent"],
                  out=(s["selected"], s["held"]), blocks=s["blocks"])
    s["cache"].attend(s["q"], s["selected"], s["held"], scale=s["scale"], out=s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"], "blocks": s["blocks"], "selected": s["selected"], "held": s["held"]}


_RUN = {"append": (_append_plain, _append_own), "read": (_read_plain_both, _read_own), "attention": (_attention_plain, _attention_own),
        "bounds": (_bounds_plain, _bounds_own), "sparse": (_sparse_plain, _sparse_own)}


# -------------------------------------------------------------------- work --
def _size(dtype):
    return 4 if dtype == "f32" else 2


def _token_bytes(case):
    """Bytes of one token's K and V in the cache."""
    return 2 * case["kv_heads"] * _block(case["dim"], case["format"]) // PAGE


def _mean_length(case):
    return 0.5 * (case["shortest"] + case["longest"])


def work(case):
    kind, d, kv = case["kind"], case["dim"], case["kv_heads"]
    values = 2 * kv * d
    if kind == "append":
        T = case["tokens"]
        return {"bytes": T * (values * (_size(case["dtype"]) + _size(case["read"])) + 2 * _token_bytes(case) + 8), "flops": 6.0 * T * values}
    if kind == "read":
        return {"bytes": case["tokens"] * (_token_bytes(case) + values * _size(case["dtype"]) + 4), "flops": 2.0 * case["tokens"] * values}
    if kind == "bounds":
        keys = case["pages"] * (PAGE if case["full"] else 0.5 * (PAGE + 1))
        return {"bytes": keys * _token_bytes(case) / 2 + case["pages"] * (kv * (2 * d + 4) + 4), "flops": 2.0 * keys * kv * d}
    rows = case["batch"] * case["q_heads"]
    mean, e = _mean_length(case), _size(case["dtype"])
    if kind == "attention":
        keys = case["batch"] * (mean if not case["window"] else min(mean, case["window"]))
        nbytes = keys * _token_bytes(case) + keys / PAGE * 4 + rows * (2 * d * e + 4)
        if case["step"]:
            nbytes += case["batch"] * (values * e + _token_bytes(case)) + 2 * rows * d * e
        return {"bytes": nbytes, "flops": 4.0 * keys * case["q_heads"] * d}
    pages = case["batch"] * mean / PAGE
    held = min(pages, case["batch"] * case["keep"])
    return {"bytes": pages * (kv * (2 * d + 4) + 4) + held * (PAGE * _token_bytes(case) + 8 * kv) + rows * (2 * d * e + 4),
            "flops": 2.0 * pages * case["q_heads"] * d + 4.0 * held * PAGE * case["q_heads"] * d}


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    """The definitions, token by token or sequence by sequence, in 64 bits."""
    s = prepare(case, seed)
    return {"append": _exact_append, "read": _exact_read, "attention": _exact_attention, "bounds": _exact_bounds,
            "sparse": _exact_sparse}[case["kind"]](case, s)


def _exact_append(case, s):
    """Each value to the nearest that its block can hold."""
    def rounded(y, lowest, highest, bits):                    # to `bits` bits behind the first, exponents from `lowest` on
        step = 2.0 ** (torch.frexp(y).exponent - 1).clamp_min(lowest).double() / 2 ** bits
        return (torch.round(y / step) * step).clamp_max(highest)

    out = {}
    for name in ("k", "v"):
        x = s[name].double()
        scale = (x.abs().amax(-1) / 2688.0).float().double()              # what is stored, in 32 and 8 bits
        x = x.reshape(*x.shape[:-1], -1, 16)
        unit = (rounded(x.abs().amax(-1) / (6.0 * scale[..., None]), -6, 448.0, 3) * scale[..., None])[..., None]
        y = torch.where(unit > 0, x.abs() / torch.where(unit > 0, unit, 1.0), 0.0)
        out[name] = (torch.sign(x) * rounded(y, 0, 6.0, 1) * unit).flatten(-2)
    return out


def _exact_read(case, s):
    k, v = (_at_slots(s["pool"], which, s["slots"].long()[:, None], torch.arange(case["kv_heads"], device="cuda")[None], case)
            for which in (0, 1))
    return {"k": k, "v": v}


def _at_slots(pool, which, slots, head, case):
    """Values of a pool at slots and heads, from its bytes, in 64 bits: [..][dim]."""
    kv, d, fmt = case["kv_heads"], case["dim"], case["format"]
    block = _block(d, fmt)
    base = (slots // PAGE) * (2 * kv * block) + (which * kv + head) * block
    place = slots % PAGE
    i = torch.arange(d, device="cuda")
    if fmt == "bf16":
        return pool.view(torch.bfloat16)[(base // 2 + place * d)[..., None] + i].double()
    scale = pool.view(torch.float32)[(base + block) // 4 - PAGE + place].double()[..., None]
    if fmt == "e2m1":
        byte = pool[(base + place * (d // 2))[..., None] + i // 2].long() >> 4 * (i % 2)
        m, e = byte & 1, byte >> 1 & 3
        size = torch.where(e > 0, (1.0 + 0.5 * m) * 2.0 ** (e - 1).double(), 0.5 * m.double())
        each = pool[(base + PAGE * (d // 2) + place * (d // 16))[..., None] + i // 16].view(torch.float8_e4m3fn).double()
        return torch.where((byte & 8) > 0, -size, size) * each * scale
    return pool[(base + place * d)[..., None] + i].view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).double() * scale


def _exact_attend(q, k, v, scale):
    """One sequence: q [kv head][group][dim], k, v [kv head][key][dim]."""
    x = torch.einsum("hgd,htd->hgt", q, k) * scale
    return torch.einsum("hgt,htd->hgd", torch.softmax(x, -1), v), torch.logsumexp(x, -1)


def _turn(x, positions):
    half = x.shape[-1] // 2
    f = torch.tensor([math.exp(-i / half * math.log(THETA)) for i in range(half)], dtype=torch.float64, device="cuda")
    a = positions.double()[:, None] * f
    z = torch.complex(x[..., :half].double(), x[..., half:].double()) * torch.polar(torch.ones_like(a), a)[:, None]
    return torch.cat([z.real, z.imag], -1)


def _exact_attention(case, s):
    B, nq, kv, d = case["batch"], case["q_heads"], case["kv_heads"], case["dim"]
    out = torch.zeros((B, nq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, nq), -math.inf, dtype=torch.float64, device="cuda")
    q = s["q"].double()
    if case["step"]:
        q = _turn(s["q"], s["positions"])
        new = _exact_append(case, {"k": _turn(s["k"], s["positions"]), "v": s["v"]})
    head = torch.arange(kv, device="cuda")[:, None]
    # a step attends with what it stored of q: its rounding belongs to the call
    asked = q.to(TORCH[case["dtype"]]).double() if case["step"] else q
    for b, n in enumerate(s["lengths"].tolist()):
        lo = max(0, n - case["window"]) if case["window"] else 0
        if n <= lo:
            continue
        at = torch.arange(lo, n, device="cuda")
        slots = s["pages"][b].long()[at // PAGE] * PAGE + at % PAGE
        k, v = (_at_slots(s["pool"], which, slots[None], head, case) for which in (0, 1))
        if case["step"]:
            k[:, -1], v[:, -1] = new["k"][b], new["v"][b]
        o, x = _exact_attend(asked[b].view(kv, nq // kv, d), k, v, s["scale"])
        out[b], lse[b] = o.reshape(nq, d), x.reshape(nq)
    return dict({"out": out, "lse": lse}, **({"q": q} if case["step"] else {}))


def _exact_bounds(case, s):
    """Scales; the codes are whole numbers of rounded scales."""
    kv = case["kv_heads"]
    scales = torch.zeros((s["bounds"].numel() // _record(kv, case["dim"]), kv), dtype=torch.float64, device="cuda")
    head = torch.arange(kv, device="cuda")[None]
    most = torch.zeros((s["last"].numel(), kv), dtype=torch.float64, device="cuda")
    for place in range(PAGE):
        slots = (s["last"].long() // PAGE * PAGE + place)[:, None]
        size = _at_slots(s["pool"], 0, slots, head, case).abs().amax(-1)
        most = torch.where(slots <= s["last"].long()[:, None], torch.maximum(most, size), most)
    scales[s["last"].long() // PAGE] = most / 127.0
    return {"codes": None, "scales": scales}


def _exact_sparse(case, s):
    """The attention in 64 bits over the pages of the highest scores, which are numbers of 32 bits by their definition."""
    B, nq, kv, d, keep = case["batch"], case["q_heads"], case["kv_heads"], case["dim"], case["keep"]
    group = nq // kv
    out = torch.zeros((B, nq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, nq), -math.inf, dtype=torch.float64, device="cuda")
    record = _record(kv, d)
    head = torch.arange(kv, device="cuda")
    f32 = np.float32
    for b, n in enumerate(s["lengths"].tolist()):
        if n <= 0:
            continue
        count = -(-n // PAGE)
        pages = s["pages"][b, :count].long()
        rows = s["bounds"].view(-1, record)[pages]
        ends = rows[:, :kv * 2 * d].contiguous().view(torch.int8).view(count, kv, 2, d).cpu().numpy().astype(np.int64)
        scales = rows[:, kv * 2 * d:kv * (2 * d + 4)].contiguous().view(torch.float32).cpu().numpy()
        q = s["q"][b].float().cpu().numpy().reshape(kv, group, d)
        slots = []
        for h in range(kv):
            best = None
            for x in q[h]:
                most = np.abs(x).max()
                whole = np.rint(x * (f32(LEVELS) / most)).astype(np.int64)
                dot = ends[:, h, 0] @ np.maximum(whole, 0) + ends[:, h, 1] @ np.minimum(whole, 0)
                t = dot.astype(f32) * most
                best = t if best is None else np.maximum(best, t)
            score = best * scales[:, h]
            forced = set(range(min(case["first"], count))) | set(range(max(0, count - case["recent"]), count))
            rest = [i for i in np.argsort(-score, kind="stable").tolist() if i not in forced]
            chosen = sorted(list(forced) + rest[:max(0, keep - len(forced))]) if count > keep else list(range(count))
            at = (torch.tensor(chosen, device="cuda")[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()
            at = at[at < n]
            slots.append(pages[at // PAGE] * PAGE + at % PAGE)
        slots = torch.stack(slots)
        k, v = (_at_slots(s["pool"], which, slots, head[:, None], case) for which in (0, 1))
        o, x = _exact_attend(s["q"][b].double().view(kv, group, d), k, v, s["scale"])
        out[b], lse[b] = o.reshape(nq, d), x.reshape(nq)
    return {"out": out, "lse": lse, "blocks": None, "selected": None, "held": None}
