"""A paged context cache filled with known keys and values, and the operators' definitions in 64 bits."""
import math

import torch

from paper_2511_18793_b200 import synth

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
#: half a step of a rounding to the type, relative to the value
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
_engines = {}


def engine(dtype, stream=None):
    """A context of the library, on the smallest model of the storage type (kept for the session unless it has a stream of its own)."""
    from paper_2511_18793_b200 import binding
    if stream is None and dtype in _engines:
        return _engines[dtype]
    w = synth.scaled(synth.WORKLOADS["tiny" if dtype == "fp32" else "small"], n_layers=1, n_items=1000, batch=1, n_hist=2, beam=2)
    cat = torch.from_numpy(synth.make_catalog(w)).cuda()
    weights = synth.make_weights(w, device="cuda")
    torch.cuda.synchronize()
    eng = binding.Engine(binding.make_config(w), weights, cat, stream=stream)
    if stream is None:
        _engines[dtype] = eng
    return eng


class Paged:
    """Sequences of the given lengths, `news` of whose last positions are new rows; what no sequence holds is `garbage`."""

    def __init__(self, dtype, news, lens, hq, hkv, hd, page, heads_outside=True, garbage=float("nan"), seed=0, tail_rows=0, extra_pages=3):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.dt = dtype, TYPES[dtype]
        self.news, self.lens, self.hq, self.hkv, self.hd, self.page = list(news), list(lens), hq, hkv, hd, page
        pages = [-(-n // page) for n in lens]
        n_pages = sum(pages) + extra_pages
        order = torch.randperm(n_pages, generator=g)[: sum(pages)].to(torch.int32)
        self.table = torch.full((len(lens), max(pages + [1])), 2 ** 30, dtype=torch.int32)     # (entries behind the end are not read)
        self.k = [torch.randn(n, hkv, hd, generator=g).to(self.dt) for n in lens]
        self.v = [torch.randn(n, hkv, hd, generator=g).to(self.dt) for n in lens]
        shape = (n_pages, hkv, page, hd) if heads_outside else (n_pages, page, hkv, hd)
        kp, vp = torch.full(shape, garbage, dtype=self.dt), torch.full(shape, garbage, dtype=self.dt)
        lk, lv = (kp, vp) if heads_outside else (kp.transpose(1, 2), vp.transpose(1, 2))
        at = 0
        for b, n in enumerate(pages):
            ids = order[at: at + n]
            self.table[b, :n] = ids
            at += n
            for t in range(self.lens[b]):
                lk[ids[t // page], :, t % page] = self.k[b][t]
                lv[ids[t // page], :, t % page] = self.v[b][t]
        self.starts = [0]
        for n in news:
            self.starts.append(self.starts[-1] + n)
        self.rows = self.starts[-1] + tail_rows
        self.q = torch.randn(max(self.rows, 1), hq, hd, generator=g).to(self.dt)[: self.rows]
        kd, vd = kp.cuda(), vp.cuda()
        self.k_pool, self.v_pool = (kd, vd) if heads_outside else (kd.transpose(1, 2), vd.transpose(1, 2))
        self.d_table = self.table.cuda()
        self.row_start = torch.tensor(self.starts, dtype=torch.int32).cuda()
        self.kv_len = torch.tensor(self.lens, dtype=torch.int32).cuda()

    def kv(self, max_new=None, max_kv=None):
        from paper_2511_18793_b200 import binding
        return binding.PagedKV(self.k_pool, self.v_pool, self.d_table, self.row_start, self.kv_len,
                               max(self.news) if max_new is None else max_new, max(self.lens) if max_kv is None else max_kv)


def reference(p, scale=None, causal=True, window=0, softcap=0.0, slopes=None, rows=None):
    """(out, lse, tolerance) in 64 bits of every new row.  Positions that a row does not see are cut out, not weighted with zero.

    Tolerance.  bf16: a weight is rounded to bf16 once (half a step of it), the result once; scores, sums and exponentials are in 32 bits,
    which a quarter of the first covers.  fp32: a score is a sum of hd products and a few steps more, off by (hd + 4) 2^-24 sum |q k| scale,
    the exponential doubles nothing but adds 2^-22 (|s| + 1); a weight is off by twice that (its own and the sum's), the sums over n positions by n 2^-24."""
    hd, g = p.hd, p.hq // p.hkv
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out = torch.zeros(p.rows, p.hq, hd, dtype=torch.float64)
    lse = torch.full((p.rows, p.hq), -math.inf, dtype=torch.float64)
    tol = torch.zeros(p.rows, p.hq, hd, dtype=torch.float64)
    q = p.q.double()
    for b, (n, length) in enumerate(zip(p.news, p.lens)):
        k, v = p.k[b].double(), p.v[b].double()
        for i in range(n):
            row = p.starts[b] + i
            if rows is not None and row not in rows:
                continue
            at = length - n + i
            hi = min(length, at + 1) if causal else length
            lo = max(0, at - window + 1) if window else 0
            if hi <= lo:
                continue
            t = torch.arange(lo, hi)
            for h in range(p.hq):
                ks, vs = k[lo:hi, h // g], v[lo:hi, h // g]
                s = (ks @ q[row, h]) * scale
                size = (ks.abs() @ q[row, h].abs()) * abs(scale)
                if softcap:
                    s = softcap * torch.tanh(s / softcap)
                bias = torch.zeros_like(s) if slopes is None else float(slopes[h]) * (at - t).abs().double()
                s = s - bias
                lse[row, h] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[row, h])
                out[row, h] = w @ vs
                spread = w @ vs.abs()
                if p.dtype == "bf16":
                    tol[row, h] = 1.25 * HALF["bf16"] * spread + HALF["bf16"] * out[row, h].abs() + 1e-6
                else:
                    delta = ((hd + 4) * 2.0 ** -24 * size + 2.0 ** -22 * (s.abs() + bias + 1)).max()
                    tol[row, h] = (2 * delta + (len(t) + 8) * 2.0 ** -24) * spread + 2.0 ** -24 * out[row, h].abs() + 1e-7
    return out, lse, tol
