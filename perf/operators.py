"""Timing cases of the operators for a paged context cache and for 8-bit projections.

A case is one call of one operator on shapes of this repository's workloads (heads, widths, beams and history lengths of
`synth.WORKLOADS`) or on generic ones:

  append    rotary embedding of a batch's new q and k rows, and their k and v appended to a paged cache
  attend    attention of the new rows (a token, a chunk, a beam set) over the paged cache
  quantize  rows to 8 bits with a scale each
  product   C = A W^T of 8-bit operands with a scale per row of A (token) and per row of W (channel)

`run` computes them in elementary torch operations, or, with `own` set, through the library's entry points.  `exact` is the
operators' definition in 64 bits.  Lengths of a ragged batch are a function of the case; values are a function of the seed.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
MAX_PAIRS_FLOPS = 1.25e12        # no drawn attention costs more than the largest listed one
MAX_PRODUCT_OPS = 1.44e12        # nor a drawn product


def listed():
    return [
        # one step of 64 requests that each add a token to their own history: the launch is the cost
        {"name": "append_token_64", "op": "append", "dtype": "bf16", "hq": 32, "hkv": 8, "hd": 128, "batch": 64, "new": 1, "ctx": 4000, "ragged": True,
         "page": 16, "rot": 128, "interleaved": False, "scaling": "none", "factor": 1.0},
        # the histories of eight requests on the 7B shape enter the cache (500 items of four codes and BOS), angles scaled for a longer context
        {"name": "append_prompt_16k", "op": "append", "dtype": "bf16", "hq": 32, "hkv": 8, "hd": 128, "batch": 8, "new": 2001, "ctx": 0, "ragged": False,
         "page": 64, "rot": 64, "interleaved": True, "scaling": "parts", "factor": 4.0},
        # the fp32 shape: three codes of a new item on top of a short history; the floor of a call
        {"name": "attend_tiny_fp32", "op": "attend", "dtype": "fp32", "hq": 4, "hkv": 4, "hd": 16, "batch": 4, "new": 3, "ctx": 61, "ragged": True,
         "page": 16, "causal": True, "window": 0, "softcap": 0.0, "slopes": False},
        # one request with a very long history, a token at a time: the context is split over the whole GPU
        {"name": "attend_token_1_32k", "op": "attend", "dtype": "bf16", "hq": 32, "hkv": 8, "hd": 64, "batch": 1, "new": 1, "ctx": 32768, "ragged": False,
         "page": 64, "causal": True, "window": 0, "softcap": 0.0, "slopes": False},
        # 64 requests of unequal history on the 7B shape, a token each: the cache is streamed
        {"name": "attend_token_64", "op": "attend", "dtype": "bf16", "hq": 32, "hkv": 8, "hd": 128, "batch": 64, "new": 1, "ctx": 4000, "ragged": True,
         "page": 16, "causal": True, "window": 0, "softcap": 0.0, "slopes": False},
        # returning users of unequal history send unequal chunks; capped scores, a distance bias and a window
        {"name": "attend_capped_ragged", "op": "attend", "dtype": "bf16", "hq": 32, "hkv": 8, "hd": 64, "batch": 32, "new": 512, "ctx": 2048, "ragged": True,
         "page": 32, "causal": True, "window": 1024, "softcap": 50.0, "slopes": True},
        # a long chunk behind a longer context: the tensor cores are the bound
        {"name": "attend_chunk_4k", "op": "attend", "dtype": "bf16", "hq": 32, "hkv": 8, "hd": 128, "batch": 1, "new": 4096, "ctx": 16384, "ragged": False,
         "page": 64, "causal": True, "window": 0, "softcap": 0.0, "slopes": False},
        # the verify rows of one request (beam 10, two levels) before a product
        {"name": "quantize_20", "op": "quantize", "dtype": "bf16", "rows": 20, "cols": 2048},
        # a prompt pass's MLP rows on the 7B shape
        {"name": "quantize_16k", "op": "quantize", "dtype": "bf16", "rows": 16008, "cols": 11008},
        # the gate/up product of one request's verify pass: bound by reading the weights
        {"name": "product_20", "op": "product", "dtype": "bf16", "rows": 20, "cols": 16384, "depth": 2048, "float_out": False, "bias": False},
        # the same of an ordinary batch on the 24-layer backbone, an odd number of rows, fp32 out with a bias
        {"name": "product_971", "op": "product", "dtype": "bf16", "rows": 971, "cols": 9728, "depth": 896, "float_out": True, "bias": True},
        # the down projection of a prompt pass on the 7B shape
        {"name": "product_16k", "op": "product", "dtype": "bf16", "rows": 16008, "cols": 4096, "depth": 11008, "float_out": False, "bias": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: query heads, KV heads, head dimension: the workloads' shapes, one query head per KV head, one KV head for all
HEADS = ((8, 8, 64), (14, 2, 64), (32, 8, 64), (12, 2, 128), (32, 8, 128), (16, 1, 128))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "attend", "quantize", "product", "product"))
    if op == "quantize":
        return {"op": op, "dtype": rng.choice(("bf16", "bf16", "fp32")), "rows": _log(rng, 1, 16008), "cols": _log(rng, 64, 11008)}
    if op == "product":
        depth, cols = 64 * _log(rng, 2, 172), 32 * _log(rng, 2, 688)
        rows = min(_log(rng, 1, 16008), int(MAX_PRODUCT_OPS / (2.0 * depth * cols)))
        return {"op": op, "dtype": "bf16", "rows": rows, "cols": cols, "depth": depth, "float_out": rng.random() < 0.3, "bias": rng.random() < 0.3}
    hq, hkv, hd = rng.choice(HEADS)
    dtype = "bf16"
    if rng.random() < 0.15:
        dtype, hq, hkv, hd = "fp32", 4, 4, 16
    page = rng.choice((16, 16, 32, 64, 128))
    case = {"op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "hd": hd, "ragged": rng.random() < 0.7, "page": page}
    if op == "append":
        case.update(new=rng.choice((1, _log(rng, 2, 2001))), ctx=_log(rng, 1, 32768))
        case["batch"] = min(_log(rng, 1, 256), max(1, 16008 // case["new"]))
        case.update(rot=rng.choice((hd, hd // 2)), interleaved=rng.random() < 0.5)
        case["scaling"] = rng.choice(("none", "linear", "parts"))
        case["factor"] = 1.0 if case["scaling"] == "none" else rng.choice((2.0, 4.0, 8.0))
        # at most 1 GB of keys and values behind the new rows
        while case["batch"] > 1 and 4.0 * case["batch"] * (case["ctx"] + case["new"]) * hkv * hd > 1e9:
            case["batch"] = max(1, case["batch"] * 2 // 3)
        return case
    kind = rng.choice(("token", "token", "chunk", "chunk", "beams"))
    case["new"] = 1 if kind == "token" else _log(rng, 2, 4096) if kind == "chunk" else rng.choice((10, 20, 30, 60, 100, 150))
    case["ctx"] = _log(rng, 16, 32768 if dtype == "bf16" else 1024)
    case["batch"] = _log(rng, 1, 128)
    case["causal"] = kind != "beams"
    case["window"] = _log(rng, 64, 4096) if kind != "beams" and rng.random() < 0.25 else 0
    case["softcap"] = 50.0 if rng.random() < 0.2 else 0.0
    case["slopes"] = rng.random() < 0.2
    if dtype == "fp32":
        case["new"], case["batch"] = min(case["new"], 64), min(case["batch"], 16)
    # at most 2 GB of keys and values, and the largest listed case's arithmetic
    while case["batch"] > 1 and (4.0 * case["batch"] * (case["ctx"] + case["new"]) * hkv * hd > 2e9 or work(case)["flops"] > MAX_PAIRS_FLOPS):
        case["batch"] = max(1, case["batch"] * 2 // 3)
    while work(case)["flops"] > MAX_PAIRS_FLOPS:
        case["ctx"] = max(16, case["ctx"] * 2 // 3)
    return case


# ----------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------

def _lengths(case):
    """New rows and context positions of each sequence."""
    b, new, ctx = case["batch"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [new] * b, [ctx] * b
    rng = random.Random(7919 * b + 31 * new + ctx)
    news = [new] + [rng.randint(max(1, new // 4), new) for _ in range(b - 1)]
    ctxs = [ctx] + [rng.randint(ctx // 4, ctx) for _ in range(b - 1)]
    return news, ctxs


def _randn(gen, *shape, dtype=torch.float32, std=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=gen)


def _paged_inputs(case, gen):
    """A pool of pages in shuffled order, its page table, and the rows that are new."""
    s = SimpleNamespace(case=case)
    s.news, s.ctxs = _lengths(case)
    dt, hq, hkv, hd, ps = TYPES[case["dtype"]], case["hq"], case["hkv"], case["hd"], case["page"]
    s.lens = [n + c for n, c in zip(s.news, s.ctxs)]
    pages = [-(-n // ps) for n in s.lens]
    n_pages = sum(pages) + 3
    order = torch.randperm(n_pages, device=DEV, generator=gen)[: sum(pages)].to(torch.int32)
    s.page_table = torch.full((case["batch"], max(pages)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(pages):
        s.page_table[b, :n] = order[at: at + n]
        at += n
    s.k_pool = _randn(gen, n_pages, hkv, ps, hd, dtype=dt)
    s.v_pool = _randn(gen, n_pages, hkv, ps, hd, dtype=dt)
    starts = [0]
    for n in s.news:
        starts.append(starts[-1] + n)
    s.starts, rows = starts, starts[-1]
    s.row_start = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s.kv_len = torch.tensor(s.lens, dtype=torch.int32, device=DEV)
    # rows as a fused QKV projection leaves them
    s.qkv = _randn(gen, rows, (hq + 2 * hkv) * hd, dtype=dt)
    return s


def _frequencies(case):
    """Rotary frequencies in 64 bits: theta = 10000, scaled for longer contexts."""
    r = case["rot"]
    f = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r)
    if case["scaling"] == "linear":
        return f / case["factor"], 1.0
    if case["scaling"] == "parts":
        # interpolated by parts: pairs that turn at least 32 times over 4096 positions as they are, those that turn at most once
        # divided by the factor, a ramp between them; the magnitude grows with the factor's logarithm
        def pair_of(turns):
            return r * math.log(4096.0 / (turns * 2.0 * math.pi)) / (2.0 * math.log(10000.0))
        lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), r - 1)
        g = ((torch.arange(r // 2, dtype=torch.float64, device=DEV) - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (1.0 - g) + f / case["factor"] * g, 0.1 * math.log(case["factor"]) + 1.0
    return f, 1.0


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    if op in ("append", "attend"):
        s = _paged_inputs(case, gen)
        if op == "attend":
            s.slopes = None
            if case["slopes"]:
                s.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / case["hq"]) for h in range(case["hq"])], device=DEV)
        return s
    s = SimpleNamespace(case=case)
    if op == "quantize":
        # activations: a few channels are much larger than the others
        s.x = _randn(gen, case["rows"], case["cols"])
        s.x *= 1.0 + 15.0 * (torch.rand(case["cols"], device=DEV, generator=gen) < 0.01)
        s.x = s.x.to(TYPES[case["dtype"]])
        return s
    m, n, k = case["rows"], case["cols"], case["depth"]
    s.a = _randn(gen, m, k).mul_(127.0 / 4.5).round_().clamp_(-127, 127).to(torch.int8)
    s.w = _randn(gen, n, k).mul_(127.0 / 4.5).round_().clamp_(-127, 127).to(torch.int8)
    s.a_scale = torch.rand(m, device=DEV, generator=gen).mul_(0.02).add_(0.03)
    s.w_scale = torch.rand(n, device=DEV, generator=gen).mul_(4e-4).add_(5e-4)
    s.bias = _randn(gen, n) if case["bias"] else None
    return s


_engines = {}


def _engine(dtype):
    """A context of the library: the smallest model of the storage type."""
    if dtype not in _engines:
        from paper_2511_18793_b200 import binding, synth
        w = synth.scaled(synth.WORKLOADS["tiny" if dtype == "fp32" else "small"], n_layers=1, n_items=1000, batch=1, n_hist=2, beam=2)
        _engines[dtype] = binding.Engine(binding.make_config(w), synth.make_weights(w, device=DEV), torch.from_numpy(synth.make_catalog(w)).to(DEV))
    return _engines[dtype]


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2511_18793_b200 import binding
        s.eng = _engine(case["dtype"])
        if case["op"] in ("append", "attend"):
            s.kv = binding.PagedKV(s.k_pool, s.v_pool, s.page_table, s.row_start, s.kv_len, max_new=max(s.news), max_kv=max(s.lens))
        if case["op"] == "append":
            rope = binding.Rope(rot_dim=case["rot"], theta=10000.0, interleaved=case["interleaved"], scaling=case["scaling"], factor=case["factor"],
                                trained_positions=4096)
            s.rope = s.eng.rope_table(rope, max(s.lens))
    if case["op"] == "append":
        s.q_out = torch.empty(s.starts[-1], case["hq"], case["hd"], dtype=TYPES[case["dtype"]], device=DEV)
    torch.cuda.synchronize()
    return s


def _split(s):
    c = s.case
    hq, hkv, hd = c["hq"], c["hkv"], c["hd"]
    x = s.qkv.view(s.starts[-1], hq + 2 * hkv, hd)
    return x[:, :hq], x[:, hq: hq + hkv], x[:, hq + hkv:]


# ----------------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------------

def run(state):
    op = state.case["op"]
    if op == "append":
        return _append_own(state) if own else _append_plain(state)
    if op == "attend":
        return _attend_own(state) if own else _attend_plain(state)
    if op == "quantize":
        return _quantize_own(state) if own else _quantize_plain(state)
    return _product_own(state) if own else _product_plain(state)


def _append_own(s):
    q, k, v = _split(s)
    s.eng.kv_append(s.kv, k, v, q=q, rope=s.rope, q_out=s.q_out)
    return s.q_out, s.k_pool, s.v_pool


def _attend_own(s):
    c = s.case
    q, _, _ = _split(s)
    return s.eng.paged_attention(s.kv, q, causal=c["causal"], window=c["window"], softcap=c["softcap"], slopes=s.slopes)


def _quantize_own(s):
    q, scale = s.eng.quantize_rows(s.x)
    return q.float() * scale[:, None], scale


def _product_own(s):
    c = s.case
    out = torch.empty(c["rows"], c["cols"], dtype=torch.float32 if c["float_out"] else TYPES[c["dtype"]], device=DEV)
    return s.eng.gemm_int8(s.a, s.a_scale, s.w, s.w_scale, out, epilogue=1 if c["float_out"] else 0, bias=s.bias)


def _slots(s):
    """Position in its sequence, page and place in the page of every new row."""
    c = s.case
    rows = torch.arange(s.starts[-1], device=DEV)
    seq = torch.searchsorted(s.row_start[1:].long(), rows, right=True)
    pos = s.kv_len.long()[seq] - s.row_start.long()[seq + 1] + rows
    page = s.page_table.long()[seq, pos // c["page"]]
    return pos, page, pos % c["page"]


def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def _append_plain(s):
    c = s.case
    q, k, v = _split(s)
    pos, page, at = _slots(s)
    f, mag = _frequencies(c)
    ang = pos.double()[:, None] * f                          # (angles of far positions: 64 bits)
    cos, sin = (torch.cos(ang) * mag).float()[:, None], (torch.sin(ang) * mag).float()[:, None]
    s.q_out.copy_(_rotate(q, cos, sin, c["rot"], c["interleaved"]).to(q.dtype))
    s.k_pool[page, :, at] = _rotate(k, cos, sin, c["rot"], c["interleaved"]).to(k.dtype)
    s.v_pool[page, :, at] = v
    return s.q_out, s.k_pool, s.v_pool


def _attend_plain(s):
    c = s.case
    hq, hkv, hd, ps = c["hq"], c["hkv"], c["hd"], c["page"]
    g = hq // hkv
    q, _, _ = _split(s)
    out = torch.empty(s.starts[-1], hq, hd, dtype=q.dtype, device=DEV)
    for b in range(c["batch"]):
        n, length = s.news[b], s.lens[b]
        r0 = s.starts[b]
        table = s.page_table[b, : -(-length // ps)].long()
        p = torch.arange(length - n, length, device=DEV)[:, None]
        j = torch.arange(length, device=DEV)[None, :]
        seen = torch.ones(n, length, dtype=torch.bool, device=DEV)
        if c["causal"]:
            seen &= j <= p
        if c["window"]:
            seen &= j > p - c["window"]
        for h in range(hkv):
            k = s.k_pool[table, h].reshape(-1, hd)[:length].float()
            v = s.v_pool[table, h].reshape(-1, hd)[:length].float()
            x = q[r0: r0 + n, h * g: (h + 1) * g].float().transpose(0, 1) @ k.T / math.sqrt(hd)
            if c["softcap"]:
                x = c["softcap"] * torch.tanh(x / c["softcap"])
            if s.slopes is not None:
                x = x - s.slopes[h * g: (h + 1) * g, None, None] * (p - j).abs()
            x = x.masked_fill_(~seen, -math.inf)
            x = torch.exp(x - x.amax(dim=-1, keepdim=True))
            x = (x @ v) / x.sum(dim=-1, keepdim=True)
            out[r0: r0 + n, h * g: (h + 1) * g] = x.transpose(0, 1).to(q.dtype)
    return out


def _quantize_plain(s):
    x = s.x.double()                                         # (a value half as large as the largest lies on a border)
    top = x.abs().amax(dim=1)
    q = torch.round(x * 127.0 / torch.where(top > 0, top, 1.0)[:, None]).to(torch.int8)
    scale = (top / 127.0).float()
    return q.float() * scale[:, None], scale


def _product_plain(s):
    c = s.case
    acc = s.a.double() @ s.w.double().T                      # whole numbers: 64 bits hold the sums exactly
    x = acc.float() * s.a_scale[:, None] * s.w_scale
    if s.bias is not None:
        x = x + s.bias
    return x if c["float_out"] else x.to(TYPES[c["dtype"]])


# ----------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------------

def _pairs(n, length, causal, window):
    """Visible (row, position) pairs of a sequence, and the positions that some row sees."""
    if not causal:
        return n * length, length
    total = 0
    first = length - n
    if not window or window >= length:
        return n * first + n * (n + 1) // 2, length
    # rows at position p see min(p + 1, window)
    short = max(0, min(n, window - 1 - first))               # rows with p + 1 < window
    total = short * (first + 1) + short * (short - 1) // 2 + (n - short) * window
    return total, length - max(0, first - window + 1)


def work(case):
    op = case["op"]
    es = 4 if case["dtype"] == "fp32" else 2
    if op in ("append", "attend"):
        news, ctxs = _lengths(case)
        rows, hq, hkv, hd = sum(news), case["hq"], case["hkv"], case["hd"]
        if op == "append":
            return {"bytes": 2 * rows * (hq + 2 * hkv) * hd * es, "flops": 3 * rows * (hq + hkv) * case["rot"]}
        pairs = seen = 0
        for n, c in zip(news, ctxs):
            a, b = _pairs(n, n + c, case["causal"], case["window"])
            pairs, seen = pairs + a, seen + b
        return {"bytes": (2 * rows * hq + 2 * seen * hkv) * hd * es, "flops": 4 * pairs * hq * hd}
    if op == "quantize":
        m, k = case["rows"], case["cols"]
        return {"bytes": m * k * (es + 1) + 4 * m, "flops": 3 * m * k}
    m, n, k = case["rows"], case["cols"], case["depth"]
    return {"bytes": m * k + n * k + m * n * (4 if case["float_out"] else es) + 4 * (m + n), "flops": 2 * m * n * k}


# ----------------------------------------------------------------------------------------------------
# the definitions, in 64 bits
# ----------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "append":
        return _append_exact(s)
    if op == "attend":
        return _attend_exact(s)
    if op == "quantize":
        x = s.x.double()
        top = torch.maximum(x.max(dim=1).values, -x.min(dim=1).values)[:, None]
        whole = torch.where(top > 0, torch.round(127.0 * x / top), torch.zeros((), dtype=torch.float64, device=DEV))
        return whole * top / 127.0, top[:, 0] / 127.0
    out = torch.empty(case["rows"], case["cols"], dtype=torch.float64, device=DEV)
    wt = s.w.double().T.contiguous()
    for i in range(0, case["rows"], 2048):
        out[i: i + 2048] = (s.a[i: i + 2048].double() @ wt) * s.a_scale[i: i + 2048].double()[:, None] * s.w_scale.double()[None, :]
    if s.bias is not None:
        out += s.bias.double()
    return out


def _append_exact(s):
    """Every pair as a complex number, turned by e^{i angle}."""
    c = s.case
    hq, hkv, hd, rot, ps = c["hq"], c["hkv"], c["hd"], c["rot"], c["page"]
    f, mag = _frequencies(c)
    rows = s.qkv.double().view(s.starts[-1], hq + 2 * hkv, hd)
    q = torch.empty(s.starts[-1], hq, hd, dtype=torch.float64, device=DEV)
    kp, vp = s.k_pool.double(), s.v_pool.double()
    first, second = ((slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot)))
    for b in range(c["batch"]):
        x = rows[s.starts[b]: s.starts[b + 1]].clone()
        p = torch.arange(s.ctxs[b], s.lens[b], device=DEV)
        turn = torch.polar(torch.full((len(p), rot // 2), mag, dtype=torch.float64, device=DEV), p.double()[:, None] * f[None, :])
        heads = x[:, : hq + hkv]
        z = torch.complex(heads[..., first].contiguous(), heads[..., second].contiguous()) * turn[:, None, :]
        heads[..., first], heads[..., second] = z.real, z.imag
        q[s.starts[b]: s.starts[b + 1]] = x[:, :hq]
        page = s.page_table[b].long()[torch.div(p, ps, rounding_mode="floor")]
        kp[page, :, p % ps] = x[:, hq: hq + hkv]
        vp[page, :, p % ps] = x[:, hq + hkv:]
    return q, kp, vp


def _attend_exact(s):
    """Row block by row block: log-sum-exp of the visible scores, then the weighted sum."""
    c = s.case
    hq, hkv, hd, ps = c["hq"], c["hkv"], c["hd"], c["page"]
    g = hq // hkv
    q = s.qkv.view(s.starts[-1], hq + 2 * hkv, hd)[:, :hq]
    out = torch.empty(s.starts[-1], hq, hd, dtype=torch.float64, device=DEV)
    for b in range(c["batch"]):
        length, n = s.lens[b], s.news[b]
        table = s.page_table[b, : (length + ps - 1) // ps].long()
        k = s.k_pool[table].double().permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :length]
        v = s.v_pool[table].double().permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :length]
        j = torch.arange(length, device=DEV)
        step = max(1, min(n, int(2e8) // max(1, length * hq)))
        for i in range(0, n, step):
            m = min(step, n - i)
            p = (length - n + i + torch.arange(m, device=DEV))[:, None]
            x = q[s.starts[b] + i: s.starts[b] + i + m].double().view(m, hkv, g, hd).permute(1, 2, 0, 3)
            z = torch.einsum("hgmd,hjd->hgmj", x, k) * hd ** -0.5
            if c["softcap"]:
                z = c["softcap"] * torch.tanh(z / c["softcap"])
            if s.slopes is not None:
                z = z - s.slopes.double().view(hkv, g, 1, 1) * (p - j).abs()
            hidden = torch.zeros(m, length, dtype=torch.bool, device=DEV)
            if c["causal"]:
                hidden |= j > p
            if c["window"]:
                hidden |= j <= p - c["window"]
            z = torch.where(hidden, torch.full((), -math.inf, dtype=torch.float64, device=DEV), z)
            w = torch.exp(z - torch.logsumexp(z, dim=-1, keepdim=True))
            out[s.starts[b] + i: s.starts[b] + i + m] = torch.einsum("hgmj,hjd->mhgd", w, v).reshape(m, hq, hd)
    return out
