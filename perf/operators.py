"""The operators of a batched decode step whose speed is measured: rotary positions, writing
keys and values into a paged cache (quantised or not), reading them back, and attention of
one new token per sequence over that cache.

A cache is a byte buffer of pages.  A page holds 16 tokens: [K|V][kv head] blocks of
[16][head_dim] values, bf16, or 8-bit codes (int8, e4m3) followed by 16 fp32 scales, one
per token: value = code * scale, scale = max |x| of the token's head / 127 (int8) or / 448
(e4m3).  A slot is page * 16 + place.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TOP = {"int8": 127.0, "e4m3": 448.0}       # the largest code


def _case(name, kind, **dims):
    return dict({"name": name, "kind": kind}, **dims)


def listed():
    return [
        # one request's next token, far into its context: q and k heads in a packed q|k|v row of the 8B shape
        _case("rope one token", "rope", tokens=1, heads=40, row_heads=48, dim=128, rot=128, dtype="bf16",
              interleaved=False, scaling="bands", far=130000, inverse=False),
        # a long prompt's chunk at the 8B shape, packed rows
        _case("rope prompt", "rope", tokens=8192, heads=40, row_heads=48, dim=128, rot=128, dtype="bf16",
              interleaved=False, scaling="none", far=8192, inverse=False),
        # the gradient of part-rotated interleaved heads in fp32, a ragged count of tokens
        _case("rope gradient", "rope", tokens=1999, heads=32, row_heads=32, dim=64, rot=32, dtype="f32",
              interleaved=True, scaling="yarn", far=60000, inverse=True),
        # a decode step's batch: q rotated, k rotated and quantised with v, one token per client
        _case("append step", "append", tokens=24, run=1, q_heads=32, kv_heads=8, dim=128, rot=128, dtype="bf16",
              format="e4m3", rope=True, scaling="bands", far=30000, read=""),
        # prompts of several clients written at once
        _case("append prompts", "append", tokens=16384, run=2731, q_heads=32, kv_heads=8, dim=128, rot=128,
              dtype="bf16", format="e4m3", rope=True, scaling="none", far=4096, read=""),
        # keys and values of an fp32 engine into an int8 cache, and back as bf16 for a dense prefill
        _case("int8 and back", "append", tokens=5003, run=1251, q_heads=0, kv_heads=8, dim=64, rot=64, dtype="f32",
              format="int8", rope=False, scaling="none", far=1, read="bf16"),
        # a cached prefix of many pages read back for a dense prefill of the next turn
        _case("read prefix", "read", tokens=30011, kv_heads=8, dim=128, dtype="bf16", format="e4m3"),
        # a single short chat: launch and latency
        _case("attention short", "attention", batch=1, shortest=200, longest=200, q_heads=32, kv_heads=8, dim=128,
              dtype="bf16", format="bf16", window=0),
        # clients of the 8B shape at ordinary lengths, among them a padding row and a first token
        _case("attention batch", "attention", batch=32, shortest=500, longest=4000, q_heads=32, kv_heads=8, dim=128,
              dtype="bf16", format="bf16", window=0),
        # two documents in a long context: the split over the length
        _case("attention long", "attention", batch=2, shortest=100001, longest=131072, q_heads=32, kv_heads=8, dim=128,
              dtype="bf16", format="bf16", window=0),
        # many clients of the 14B shape (five query heads to a KV head) on an int8 cache
        _case("attention int8", "attention", batch=64, shortest=1000, longest=8192, q_heads=40, kv_heads=8, dim=128,
              dtype="bf16", format="int8", window=0),
        # the 1B shape in fp32 over an e4m3 cache with a sliding window
        _case("attention e4m3 window", "attention", batch=48, shortest=300, longest=16000, q_heads=32, kv_heads=8,
              dim=64, dtype="f32", format="e4m3", window=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "append", "read", "attention", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    dim = rng.choice([64, 128])
    scaling = rng.choice(["none", "linear", "bands", "yarn"])
    if kind == "rope":
        d = rng.choice([32, 64, 80, 96, 128, 256])
        heads = rng.randint(1, 40)
        return _unnamed(kind, tokens=_log(rng, 1, 8192), heads=heads, row_heads=heads + rng.choice([0, 0, 8]), dim=d,
                        rot=rng.choice([d, d, d // 2, d - 2 * rng.randint(0, d // 4)]), dtype=dtype,
                        interleaved=rng.random() < 0.4, scaling=scaling, far=_log(rng, 1, 1000000),
                        inverse=rng.random() < 0.3)
    fmt = rng.choice(["bf16", "int8", "e4m3"])
    kv = rng.choice([1, 2, 4, 8])
    if kind == "append":
        tokens = _log(rng, 1, 16384)
        rope = rng.random() < 0.6
        return _unnamed(kind, tokens=tokens, run=rng.randint(1, tokens), q_heads=kv * rng.choice([1, 3, 4, 5, 8]) if rope else 0,
                        kv_heads=kv, dim=dim, rot=rng.choice([dim, dim, dim // 2]), dtype=dtype, format=fmt, rope=rope,
                        scaling=scaling, far=_log(rng, 1, 200000),
                        read="bf16" if fmt == "int8" else rng.choice(["", "bf16"]))
    if kind == "read":
        return _unnamed(kind, tokens=_log(rng, 1, 30000), kv_heads=kv, dim=dim, dtype=dtype, format=fmt)
    batch = _log(rng, 1, 96)
    longest = _log(rng, 1, min(131072, 200000 // batch))
    return _unnamed(kind, batch=batch, shortest=_log(rng, 1, longest), longest=longest,
                    q_heads=kv * rng.choice([1, 2, 4, 5, 7, 8, 16]), kv_heads=kv, dim=dim, dtype=dtype, format=fmt,
                    window=rng.choice([0, 0, 0, rng.randint(1, 5000)]))


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


def _spec(case):
    """The rope's numbers: theta and the scaling rule's."""
    low, high = (1.0, 4.0) if case["scaling"] == "bands" else (1.0, 32.0)
    return {"head_dim": case["dim"], "rot_dim": case["rot"], "interleaved": case.get("interleaved", False),
            "theta": 5e5, "scaling": case["scaling"], "factor": 1.0 if case["scaling"] == "none" else 8.0,
            "original_len": 8192, "low": low, "high": high}


def _parts(pool, kv_heads, dim, fmt):
    """Views of a pool: the values or codes [page][K|V][head][16][dim] and the scales [page][K|V][head][16] (None in bf16)."""
    if fmt == "bf16":
        return pool.view(torch.bfloat16).view(-1, 2, kv_heads, PAGE, dim), None
    blocks = pool.view(-1, 2, kv_heads, PAGE * dim + 4 * PAGE)
    codes = blocks[..., :PAGE * dim].unflatten(-1, (PAGE, dim))
    return codes, blocks.view(torch.float32)[..., PAGE * dim // 4:]


def _pool(pages, kv_heads, dim, fmt, fill):
    block = PAGE * dim * 2 if fmt == "bf16" else PAGE * dim + 4 * PAGE
    return torch.full((pages * 2 * kv_heads * block,), fill, dtype=torch.uint8, device="cuda")


def _filled(g, pages, kv_heads, dim, fmt):
    """A pool as earlier calls left it: every slot holds a token."""
    pool = _pool(pages, kv_heads, dim, fmt, 0)
    values, scales = _parts(pool, kv_heads, dim, fmt)
    step = max(1, (1 << 26) // (2 * kv_heads * PAGE * dim))
    gain = torch.exp(0.6 * _normal(g, 2, kv_heads, 1, dim))
    gain[1] = 1.0
    for a in range(0, pages, step):
        n = min(step, pages - a)
        x = _normal(g, n, 2, kv_heads, PAGE, dim).mul_(gain)
        if fmt == "bf16":
            values[a:a + n] = x.to(torch.bfloat16)
            continue
        s = x.abs().amax(-1) / TOP[fmt]
        x = x.div_(s.unsqueeze(-1))
        x = x.round_().to(torch.int8) if fmt == "int8" else x.clamp_(-448, 448).to(torch.float8_e4m3fn)
        values[a:a + n] = x.view(torch.uint8)
        scales[a:a + n] = s
    return pool


def prepare(case, seed):
    g = _generator(seed, 17)
    kind = case["kind"]
    if kind == "rope":
        T, H, R, d = case["tokens"], case["heads"], case["row_heads"], case["dim"]
        rows = _normal(g, T, R, d).to(TORCH[case["dtype"]])
        first = int(_ints(g, 0, max(0, case["far"] - T), 1))
        return {"case": case, "spec": _spec(case), "x": rows[:, :H], "positions": torch.arange(first, first + T, device="cuda", dtype=torch.int32),
                "y": torch.zeros((T, H, d), dtype=rows.dtype, device="cuda")}
    if kind == "attention":
        B, kv, d = case["batch"], case["kv_heads"], case["dim"]
        lengths = _ints(g, case["shortest"], case["longest"], B)
        if B > 8:
            lengths[0], lengths[1], lengths[2] = 0, 1, case["longest"]       # a padding row and a first token
        most = -(-case["longest"] // PAGE)
        need = ((lengths + PAGE - 1) // PAGE).tolist()
        total = sum(need) + 3
        pool = _filled(g, total, kv, d, case["format"])
        order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        pages = torch.full((B, most), -1, dtype=torch.int32, device="cuda")    # entries past a length name no page
        at = 0
        for b, n in enumerate(need):
            pages[b, :n] = order[at:at + n]
            at += n
        return {"case": case, "pool": pool, "pages": pages, "lengths": lengths, "scale": d ** -0.5,
                "q": (2.0 * _normal(g, B, case["q_heads"], d)).to(TORCH[case["dtype"]]),
                "out": torch.zeros((B, case["q_heads"], d), dtype=TORCH[case["dtype"]], device="cuda"),
                "lse": torch.zeros((B, case["q_heads"]), device="cuda")}
    T, kv, d = case["tokens"], case["kv_heads"], case["dim"]
    pages = -(-T // PAGE) + 2
    if kind == "read":
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        at = torch.arange(T, device="cuda")
        slots = order[at // PAGE] * PAGE + (at % PAGE).to(torch.int32)
        return {"case": case, "pool": _filled(g, pages, kv, d, case["format"]), "slots": slots,
                "k": torch.zeros((T, kv, d), dtype=TORCH[case["dtype"]], device="cuda"),
                "v": torch.zeros((T, kv, d), dtype=TORCH[case["dtype"]], device="cuda")}
    # tokens of several sequences, `run` of each: every run starts on a page of its own and at a position of its own
    run_, nq = case["run"], case["q_heads"]
    runs = -(-T // run_)
    per = -(-run_ // PAGE)
    order = torch.randperm(runs * per, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(T, device="cuda")
    seq, off = at // run_, at % run_
    slots = order[seq * per + off // PAGE] * PAGE + (off % PAGE).to(torch.int32)
    first = _ints(g, 0, case["far"], runs)
    heads = nq + 2 * kv
    rows = _keys(g, T, heads, d).to(TORCH[case["dtype"]])                  # the packed q|k|v rows of a projection
    s = {"case": case, "spec": _spec(case), "pool": _pool(runs * per, kv, d, case["format"], 0), "slots": slots,
         "positions": first[seq] + off.to(torch.int32), "q": rows[:, :nq], "k": rows[:, nq:nq + kv], "v": rows[:, nq + kv:]}
    s["q_out"] = torch.zeros((T, nq, d), dtype=rows.dtype, device="cuda")
    if case["read"]:
        s["back"] = [torch.zeros((T, kv, d), dtype=TORCH[case["read"]], device="cuda") for _ in range(2)]
    return s


# --------------------------------------------------------------------- run --
def run(s):
    return _RUN[s["case"]["kind"]][1 if own else 0](s)


def _frequencies(spec):
    """Radians a position, in 64 bits, and the gain of the rotated values."""
    rot, theta, factor, length = spec["rot_dim"], spec["theta"], spec["factor"], spec["original_len"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    f = theta ** (-2.0 * i / rot)
    if spec["scaling"] == "linear":
        return f / factor, 1.0
    if spec["scaling"] == "bands":
        turns = length * f / (2.0 * math.pi)                                # turns within the original length
        mix = ((turns - spec["low"]) / (spec["high"] - spec["low"])).clamp(0.0, 1.0)
        return f * ((1.0 - mix) / factor + mix), 1.0
    if spec["scaling"] == "yarn":
        at = lambda turns: rot * math.log(length / (turns * 2.0 * math.pi)) / (2.0 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(at(spec["high"])), 0), min(math.ceil(at(spec["low"])), rot - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        return f / factor * ramp + f * (1.0 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _rotated(x, positions, spec, inverse=False):
    """x [tokens][heads][dim] rotated, in 32 bits (angles in 64)."""
    f, gain = _frequencies(spec)
    a = (positions.double().unsqueeze(1) * f).unsqueeze(1)
    c, n = (gain * torch.cos(a)).float(), (gain * torch.sin(a)).float()
    n = -n if inverse else n
    x, rot = x.float(), spec["rot_dim"]
    y = x.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if spec["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., first] = x[..., first] * c - x[..., second] * n
    y[..., second] = x[..., first] * n + x[..., second] * c
    return y


def _rope_plain(s):
    case = s["case"]
    s["y"].copy_(_rotated(s["x"], s["positions"], s["spec"], case["inverse"]))
    return s["y"]


def _write_plain(pool, which, x, slots, case):
    values, scales = _parts(pool, case["kv_heads"], case["dim"], case["format"])
    slots = slots.long()
    page, place = slots // PAGE, slots % PAGE
    if scales is None:
        values[page, which, :, place] = x.to(torch.bfloat16)
        return
    x = x.double()                                                          # codes next to a border
    scale = (x.abs().amax(-1) / TOP[case["format"]]).float()
    c = x / scale.double().clamp_min(1e-300).unsqueeze(-1)
    c = c.round().clamp(-127, 127).to(torch.int8) if case["format"] == "int8" else c.clamp(-448, 448).to(torch.float8_e4m3fn)
    values[page, which, :, place] = c.view(torch.uint8)
    scales[page, which, :, place] = scale


def _values(pool, case):
    """Every value of a pool in 32 bits: [page][K|V][head][16][dim]."""
    values, scales = _parts(pool, case["kv_heads"], case["dim"], case["format"])
    if scales is None:
        return values.float()
    kind = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    return values.view(kind).float() * scales.unsqueeze(-1)


def _read_plain(pool, which, slots, out, case):
    values, scales = _parts(pool, case["kv_heads"], case["dim"], case["format"])
    slots = slots.long()
    page, place = slots // PAGE, slots % PAGE
    x = values[page, which, :, place]
    if scales is not None:
        x = x.contiguous().view(torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn).float() * scales[page, which, :, place].unsqueeze(-1)
    out.copy_(x)


def _stored(s):
    """What an append wrote: the values read back, or the cache itself as the codes stand (and their scales)."""
    case = s["case"]
    out = {"q": s["q_out"]} if case["rope"] else {}
    if case["read"]:
        return dict(out, k=s["back"][0], v=s["back"][1])
    values, scales = _parts(s["pool"], case["kv_heads"], case["dim"], case["format"])
    return dict(out, cache=values) if scales is None else dict(out, cache=values.view(torch.float8_e4m3fn), scales=scales)


def _append_plain(s):
    case = s["case"]
    k, v = s["k"].float(), s["v"].float()
    if case["rope"]:
        s["q_out"].copy_(_rotated(s["q"], s["positions"], s["spec"]))
        k = _rotated(s["k"], s["positions"], s["spec"])
    _write_plain(s["pool"], 0, k, s["slots"], case)
    _write_plain(s["pool"], 1, v, s["slots"], case)
    if case["read"]:
        _read_plain(s["pool"], 0, s["slots"], s["back"][0], case)
        _read_plain(s["pool"], 1, s["slots"], s["back"][1], case)
    return _stored(s)


def _read_plain_both(s):
    _read_plain(s["pool"], 0, s["slots"], s["k"], s["case"])
    _read_plain(s["pool"], 1, s["slots"], s["v"], s["case"])
    return {"k": s["k"], "v": s["v"]}


def _attention_plain(s):
    case = s["case"]
    B, nq, kv, d = case["batch"], case["q_heads"], case["kv_heads"], case["dim"]
    values, scales = _parts(s["pool"], kv, d, case["format"])
    pages = s["pages"].long()
    L = pages.shape[1] * PAGE
    at = torch.arange(L, device="cuda")
    n = s["lengths"].unsqueeze(1)
    valid = at < n
    if case["window"]:
        valid &= at >= n - case["window"]

    def dense(which):                                                       # [batch][head][key][dim]
        x = values[pages, which]
        if scales is None:
            x = x.float()
        else:
            x = x.contiguous().view(torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn).float() * scales[pages, which].unsqueeze(-1)
        return x.transpose(1, 2).reshape(B, kv, L, d)

    q = s["q"].float().view(B, kv, nq // kv, d)
    k = dense(0)
    x = (q @ k.transpose(2, 3)) * s["scale"]
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


# ---- the framework's operators ----
_ops = None


def _kept(s, name, make):
    """The plan or cache handle that a program makes once for its shapes."""
    global _ops
    if _ops is None:
        from paper_2608_24204_gb300 import ops
        _ops = ops
    if name not in s:
        s[name] = make()
    return s[name]


def _rope_of(s):
    return _kept(s, "rope plan", lambda: _ops.Rope(**s["spec"]))


def _cache_of(s):
    case = s["case"]
    return _kept(s, "cache", lambda: _ops.PagedKV(case["kv_heads"], case["dim"], case["format"], data=s["pool"]))


def _rope_own(s):
    _rope_of(s).apply(s["x"], s["positions"], out=s["y"], inverse=s["case"]["inverse"])
    return s["y"]


def _append_own(s):
    cache = _cache_of(s)
    if s["case"]["rope"]:
        cache.append(s["k"], s["v"], s["slots"], rope=_rope_of(s), positions=s["positions"], q=s["q"], q_out=s["q_out"])
    else:
        cache.append(s["k"], s["v"], s["slots"])
    if s["case"]["read"]:
        cache.read(s["slots"], out=s["back"])
    return _stored(s)


def _read_own(s):
    _cache_of(s).read(s["slots"], out=(s["k"], s["v"]))
    return {"k": s["k"], "v": s["v"]}


def _attention_own(s):
    _cache_of(s).attend(s["q"], s["pages"], s["lengths"], scale=s["scale"], window=s["case"]["window"], out=s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


_RUN = {"rope": (_rope_plain, _rope_own), "append": (_append_plain, _append_own), "read": (_read_plain_both, _read_own),
        "attention": (_attention_plain, _attention_own)}


# -------------------------------------------------------------------- work --
def _size(dtype):
    return 4 if dtype == "f32" else 2


def _token_bytes(case):
    """Bytes of one token's K and V in the cache."""
    per = 2 * case["dim"] if case["format"] == "bf16" else case["dim"] + 4
    return 2 * case["kv_heads"] * per


def work(case):
    kind = case["kind"]
    if kind == "rope":
        n = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * _size(case["dtype"]) + 4 * case["tokens"], "flops": 3.0 * case["tokens"] * case["heads"] * case["rot"]}
    if kind == "append":
        T, e = case["tokens"], _size(case["dtype"])
        values = 2 * case["kv_heads"] * case["dim"]
        q = case["q_heads"] * case["dim"] if case["rope"] else 0
        nbytes = T * (values * e + _token_bytes(case) + 2 * q * e + 4 + (4 if case["rope"] else 0))
        if case["read"]:
            nbytes += T * (_token_bytes(case) + values * _size(case["read"]) + 4)
        return {"bytes": nbytes, "flops": T * (3.0 * values + 3.0 * q)}
    if kind == "read":
        values = 2 * case["kv_heads"] * case["dim"]
        return {"bytes": case["tokens"] * (_token_bytes(case) + values * _size(case["dtype"]) + 4), "flops": 1.0 * case["tokens"] * values}
    mean = 0.5 * (case["shortest"] + case["longest"])
    keys = case["batch"] * (mean if not case["window"] else min(mean, case["window"]))
    rows = case["batch"] * case["q_heads"]
    return {"bytes": keys * _token_bytes(case) + keys / PAGE * 4 + rows * (2 * case["dim"] * _size(case["dtype"]) + 4),
            "flops": 4.0 * keys * case["q_heads"] * case["dim"]}


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    """The definitions, token by token or sequence by sequence, in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        return _turn(s["x"], s["positions"], s["spec"], -1.0 if case["inverse"] else 1.0)
    if kind == "append":
        return _exact_append(case, s)
    if kind == "read":
        k, v = (_at_slots(s["pool"], which, s["slots"], case) for which in (0, 1))
        return {"k": k, "v": v}
    return _exact_attention(case, s)


def _turn(x, positions, spec, sign):
    """Each pair as a complex number times g exp(i sign p f)."""
    rot, x = spec["rot_dim"], x.double()
    half = rot // 2
    f, gain = [], 1.0
    for i in range(half):
        w = math.exp(-2.0 * i / rot * math.log(spec["theta"]))
        if spec["scaling"] == "linear":
            w /= spec["factor"]
        elif spec["scaling"] == "bands":
            wave = 2.0 * math.pi / w
            if wave > spec["original_len"] / spec["low"]:
                w /= spec["factor"]
            elif wave >= spec["original_len"] / spec["high"]:
                t = (spec["original_len"] / wave - spec["low"]) / (spec["high"] - spec["low"])
                w = (1.0 - t) * w / spec["factor"] + t * w
        elif spec["scaling"] == "yarn":
            d = [rot * math.log(spec["original_len"] / (2.0 * math.pi * b)) / (2.0 * math.log(spec["theta"])) for b in (spec["high"], spec["low"])]
            a, b = max(math.floor(d[0]), 0), min(math.ceil(d[1]), rot - 1)
            t = min(max((i - a) / max(b - a, 1e-3), 0.0), 1.0)
            w = w * (1.0 - t) + w / spec["factor"] * t
            gain = 0.1 * math.log(spec["factor"]) + 1.0
        f.append(w)
    a = sign * positions.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(a, gain), a)[:, None]
    if spec["interleaved"]:
        z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], half, 2).contiguous()) * turn
        head = torch.view_as_real(z).reshape(*x.shape[:-1], rot)
    else:
        z = torch.complex(x[..., :half].contiguous(), x[..., half:rot].contiguous()) * turn
        head = torch.cat([z.real, z.imag], -1)
    return torch.cat([head, x[..., rot:]], -1)


def _exact_append(case, s):
    kv, d, fmt = case["kv_heads"], case["dim"], case["format"]
    k, v = s["k"].double(), s["v"].double()
    out = {}
    if case["rope"]:
        out["q"] = _turn(s["q"], s["positions"], s["spec"], 1.0)
        k = _turn(s["k"], s["positions"], s["spec"], 1.0)
    scales, codes = [], []
    for x in (k, v):
        if fmt == "bf16":
            scales.append(None)
            codes.append(x.to(torch.bfloat16).double() if case["read"] else x)
            continue
        scale = x.abs().max(dim=-1, keepdim=True).values / TOP[fmt]
        c = torch.where(scale > 0, x / torch.where(scale > 0, scale, torch.ones_like(scale)), torch.zeros_like(x))
        c = torch.round(c) if fmt == "int8" else c.to(torch.float8_e4m3fn).double()
        scales.append(scale.squeeze(-1))
        codes.append(c if not case["read"] else c * scale)
    if case["read"]:
        return dict(out, k=codes[0], v=codes[1])
    pages = s["pool"].numel() // (2 * kv * (PAGE * d * 2 if fmt == "bf16" else PAGE * d + 4 * PAGE))
    slots = s["slots"].long()
    values = torch.zeros((pages * PAGE, 2, kv, d), dtype=torch.float64, device="cuda")
    for which in (0, 1):
        values[slots, which] = codes[which]
    out["cache"] = values.view(pages, PAGE, 2, kv, d).permute(0, 2, 3, 1, 4).contiguous()
    if fmt != "bf16":
        kept = torch.zeros((pages * PAGE, 2, kv), dtype=torch.float64, device="cuda")
        for which in (0, 1):
            kept[slots, which] = scales[which]
        out["scales"] = kept.view(pages, PAGE, 2, kv).permute(0, 2, 3, 1).contiguous()
    return out


def _at_slots(pool, which, slots, case):
    """Values of a pool at slots, from its bytes, in 64 bits: [slot][head][dim]."""
    kv, d = case["kv_heads"], case["dim"]
    block = PAGE * d * 2 if case["format"] == "bf16" else PAGE * d + 4 * PAGE
    slots = slots.long()
    base = (slots // PAGE)[:, None] * (2 * kv * block) + (which * kv + torch.arange(kv, device="cuda"))[None] * block
    place = (slots % PAGE)[:, None]
    if case["format"] == "bf16":
        at = (base // 2 + place * d)[..., None] + torch.arange(d, device="cuda")
        return pool.view(torch.bfloat16)[at].double()
    at = (base + place * d)[..., None] + torch.arange(d, device="cuda")
    codes = pool[at].view(torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn).double()
    return codes * pool.view(torch.float32)[(base + PAGE * d) // 4 + place].double()[..., None]


def _exact_attention(case, s):
    B, nq, kv, d = case["batch"], case["q_heads"], case["kv_heads"], case["dim"]
    out = torch.zeros((B, nq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, nq), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lengths"].tolist()):
        lo = max(0, n - case["window"]) if case["window"] else 0
        if n <= lo:
            continue
        at = torch.arange(lo, n, device="cuda")
        slots = s["pages"][b].long()[at // PAGE] * PAGE + at % PAGE
        q = s["q"][b].double().view(kv, nq // kv, d)
        x = torch.einsum("hgd,thd->hgt", q, _at_slots(s["pool"], 0, slots, case)) * s["scale"]
        lse[b] = torch.logsumexp(x, -1).reshape(nq)
        out[b] = torch.einsum("hgt,thd->hgd", torch.softmax(x, -1), _at_slots(s["pool"], 1, slots, case)).reshape(nq, d)
    return {"out": out, "lse": lse}
