"""The operators as a decoder uses them: 8-bit projections, rotary append to the cache, attention over it; two layers, a chunk of a prompt and
tokens behind it.  Every step is compared with its definition on what the step before really left."""
from types import SimpleNamespace

import pytest
import torch

from paged_helpers import HALF, engine, reference
from test_gpu_int8 import quantized
from test_gpu_kv_append import turned

pytestmark = pytest.mark.gpu

HQ, HKV, PAGE, LAYERS = 8, 2, 16, 2


def weights(n, k, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8).cuda(), (torch.rand(n, generator=g) * 2e-3 / k ** 0.5 + 1e-4).cuda()


def projected(q, s, w, ws):
    """The definition: the exact sum of whole numbers to 32 bits, times one scale, times the other, each a rounding to 32 bits, then bf16."""
    acc = (q.double() @ w.double().T).float()
    return ((acc * s[:, None]) * ws[None]).bfloat16()


class Layer:
    def __init__(self, hd, seed, n_pages):
        d = HQ * hd
        self.qkv, self.qkv_s = weights((HQ + 2 * HKV) * hd, d, seed)
        self.o, self.o_s = weights(d, d, seed + 1)
        self.k = torch.full((n_pages, HKV, PAGE, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.v = torch.full_like(self.k, float("nan"))


@pytest.mark.parametrize("hd,own_stream", [(64, False), (128, True)])
def test_a_prompt_and_tokens_behind_it(hd, own_stream):
    from paper_2511_18793_b200 import binding
    stream = torch.cuda.Stream() if own_stream else None
    eng = engine("bf16", stream=stream)
    d, heads = HQ * hd, HQ + 2 * HKV
    steps = [[70, 33, 0], [1, 3, 40], [1, 0, 1], [2, 1, 1]]
    lens = [0, 0, 0]
    pages = [-(-sum(s[b] for s in steps) // PAGE) for b in range(3)]
    order = torch.randperm(sum(pages) + 2, generator=torch.Generator().manual_seed(3)).to(torch.int32)
    table = torch.full((3, max(pages)), 2 ** 30, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at: at + n]
        at += n
    d_table = table.cuda()
    layers = [Layer(hd, 10 * i, len(order)) for i in range(LAYERS)]
    rope = binding.Rope(hd, scaling="parts", factor=4.0, trained_positions=64)
    tab = eng.rope_table(rope, 256)
    g = torch.Generator().manual_seed(1)
    for news in steps:
        lens = [l + n for l, n in zip(lens, news)]
        starts = [0]
        for n in news:
            starts.append(starts[-1] + n)
        rows = starts[-1]
        pos = torch.cat([torch.arange(l - n, l) for n, l in zip(news, lens)])
        x = torch.randn(rows, d, generator=g).bfloat16().cuda()
        row_start, kv_len = torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
        torch.cuda.synchronize()
        for layer in layers:
            kv = binding.PagedKV(layer.k, layer.v, d_table, row_start, kv_len, max(news), max(lens))
            # the run: nothing waits between the calls
            q8, s8 = eng.quantize_rows(x)
            qkv = torch.empty(rows, heads * hd, dtype=torch.bfloat16, device="cuda")
            if stream is not None:
                qkv.record_stream(stream)
            eng.gemm_int8(q8, s8, layer.qkv, layer.qkv_s, qkv)
            fused = qkv.view(rows, heads, hd)
            q = eng.kv_append(kv, fused[:, HQ: HQ + HKV], fused[:, HQ + HKV:], q=fused[:, :HQ], rope=tab)
            out = eng.paged_attention(kv, q)
            o8, os8 = eng.quantize_rows(out.view(rows, d))
            y = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
            if stream is not None:
                y.record_stream(stream)
            eng.gemm_int8(o8, os8, layer.o, layer.o_s, y)
            eng.sync()
            # each step by its definition
            want_q, _ = quantized(x)
            assert torch.equal(q8, want_q) and torch.equal(qkv, projected(q8, s8, layer.qkv, layer.qkv_s))
            host = fused.double().cpu()
            for got, src in ((q, host[:, :HQ]), (None, host[:, HQ: HQ + HKV])):
                want, size = turned(src, pos, rope)
                if got is None:                          # the keys are in the cache
                    got = torch.cat([torch.stack([layer.k[int(table[b, t // PAGE]), :, t % PAGE] for t in range(lens[b] - news[b], lens[b])])
                                     for b in range(3) if news[b]])
                # cosine, sine, two products and a sum in 32 bits, then the storage type's rounding
                assert bool(((got.double().cpu() - want).abs() <= HALF["bf16"] * want.abs() + 4 * 2.0 ** -24 * size).all())
            cache = SimpleNamespace(dtype="bf16", news=news, lens=lens, hq=HQ, hkv=HKV, hd=hd, rows=rows, starts=starts, q=q.cpu(), k=[], v=[])
            for b in range(3):
                for pool, into in ((layer.k, cache.k), (layer.v, cache.v)):
                    into.append(torch.stack([pool[int(table[b, t // PAGE]), :, t % PAGE] for t in range(lens[b])]).cpu() if lens[b] else torch.zeros(0, HKV, hd))
            for b in range(3):                           # (V goes in as it is)
                assert torch.equal(cache.v[b][lens[b] - news[b]:].double(), host[starts[b]: starts[b + 1], HQ + HKV:])
            want, _, tol = reference(cache)
            assert bool(((out.double().cpu() - want).abs() <= tol).all())
            assert torch.equal(o8, quantized(out.view(rows, d))[0]) and torch.equal(y, projected(o8, os8, layer.o, layer.o_s))
            x = (x.float() + y.float()).bfloat16()
            torch.cuda.synchronize()
    # what no sequence holds is as it was
    used = torch.zeros(len(order), PAGE, dtype=torch.bool)
    for b in range(3):
        for t in range(lens[b]):
            used[int(table[b, t // PAGE]), t % PAGE] = True
    for layer in layers:
        assert bool(torch.isnan(layer.k.cpu().transpose(1, 2)[~used]).all()) and bool(torch.isnan(layer.v.cpu().transpose(1, 2)[~used]).all())


def test_a_captured_step_of_two_layers():
    """One token of each sequence through the chain from a graph, again and again as the lengths grow: the same bits as eager calls."""
    from paper_2511_18793_b200 import binding
    hd, batch = 64, 3
    d, heads = HQ * hd, HQ + 2 * HKV
    stream = torch.cuda.Stream()
    eng = engine("bf16", stream=stream)
    table = torch.arange(batch * 8, dtype=torch.int32).view(batch, 8).cuda()
    start_len = torch.tensor([5, 64, 100], dtype=torch.int32)
    rope = binding.Rope(hd)

    def build():
        g = torch.Generator().manual_seed(0)
        layers = [Layer(hd, 7 * i, batch * 8) for i in range(LAYERS)]
        for layer in layers:
            layer.k.copy_(torch.randn(layer.k.shape, generator=g).bfloat16())
            layer.v.copy_(torch.randn(layer.v.shape, generator=g).bfloat16())
        return layers, start_len.clone().cuda(), torch.randn(batch, d, generator=g).bfloat16().cuda()

    tab = eng.rope_table(rope, 8 * PAGE)
    row_start = torch.arange(batch + 1, dtype=torch.int32).cuda()

    def step(layers, kv_len, x):
        for layer in layers:
            kv = binding.PagedKV(layer.k, layer.v, table, row_start, kv_len, 1, 8 * PAGE)
            q8, s8 = eng.quantize_rows(x)
            qkv = eng.gemm_int8(q8, s8, layer.qkv, layer.qkv_s, torch.empty(batch, heads * hd, dtype=torch.bfloat16, device="cuda")).view(batch, heads, hd)
            q = eng.kv_append(kv, qkv[:, HQ: HQ + HKV], qkv[:, HQ + HKV:], q=qkv[:, :HQ], rope=tab)
            o8, os8 = eng.quantize_rows(eng.paged_attention(kv, q).view(batch, d))
            x = eng.gemm_int8(o8, os8, layer.o, layer.o_s, torch.empty(batch, d, dtype=torch.bfloat16, device="cuda")) + x
        return x

    runs = []
    for captured in (False, True):
        layers, kv_len, x = build()
        torch.cuda.synchronize()
        outs = []
        with torch.cuda.stream(stream):
            if captured:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=stream):
                    y = step(layers, kv_len, x)
            for _ in range(6):
                kv_len += 1
                if captured:
                    g.replay()
                    outs.append(y.clone())
                else:
                    outs.append(step(layers, kv_len, x))
        eng.sync()
        runs.append((outs, layers))
    for a, b in zip(runs[0][0], runs[1][0]):
        assert torch.equal(a, b)
    for a, b in zip(runs[0][1], runs[1][1]):
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
