"""Attention over a paged context cache against its definition in 64 bits."""
import math

import pytest
import torch

from paged_helpers import Paged, engine, reference

pytestmark = pytest.mark.gpu


def check(p, form=None, lse=True, rows=None, eng=None, **bounds):
    form = form or {}
    eng = eng or engine(p.dtype)
    q = p.q.cuda()
    got_lse = torch.full((p.rows, p.hq), 7.0, device="cuda") if lse else None
    dev = {k: v.cuda() if torch.is_tensor(v) else v for k, v in form.items()}
    out = torch.full((p.rows, p.hq, p.hd), 5.0, dtype=p.dt, device="cuda")
    eng.paged_attention(p.kv(**bounds), q, out=out, lse=got_lse, **dev)
    eng.sync()
    want, want_lse, tol = reference(p, rows=rows, **form)
    used = slice(0, p.starts[-1]) if rows is None else sorted(rows)
    err = (out.double().cpu() - want).abs()[used]
    assert bool((err <= tol[used]).all()), float((err - tol[used]).max())
    if lse:
        g, w = got_lse.double().cpu()[used], want_lse[used]
        assert torch.equal(torch.isneginf(g), torch.isneginf(w))
        live = ~torch.isneginf(w)
        assert bool(((g - w).abs()[live] <= 2e-5 * (1 + w.abs()[live])).all())
    # rows behind the last sequence are left alone
    assert bool((out[p.starts[-1]:] == 5.0).all())
    if lse:
        assert bool((got_lse[p.starts[-1]:] == 7.0).all())
    return out


NEWS = [1, 0, 3, 17, 1, 2]
LENS = [1, 5, 3, 90, 129, 64]


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("fp32", 4, 4, 16), ("fp32", 6, 2, 32), ("fp32", 8, 2, 64), ("fp32", 3, 1, 128), ("bf16", 4, 2, 16),
                                             ("bf16", 4, 4, 32), ("bf16", 8, 8, 64), ("bf16", 14, 2, 64), ("bf16", 12, 2, 128), ("bf16", 16, 1, 128)])
@pytest.mark.parametrize("page", [1, 5, 16, 24, 64])
def test_types_heads_and_pages(dtype, hq, hkv, hd, page):
    check(Paged(dtype, NEWS, LENS, hq, hkv, hd, page, heads_outside=page % 2 == 0, tail_rows=2))


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("form", [dict(causal=False), dict(window=1), dict(window=9), dict(window=70), dict(softcap=20.0, scale=0.3),
                                  dict(slopes="yes"), dict(causal=False, slopes="yes", softcap=5.0), dict(window=33, slopes="yes", softcap=30.0)])
def test_forms(dtype, hd, form):
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = torch.tensor([2.0 ** -(h + 1) for h in range(8)])
    check(Paged(dtype, [4, 1, 30, 7], [4, 200, 131, 65], 8, 2, hd, 16), form)


@pytest.mark.parametrize("dtype,hd,heads_outside", [("bf16", 128, True), ("bf16", 64, False), ("fp32", 16, True)])
@pytest.mark.parametrize("form", [dict(), dict(causal=False), dict(window=100)])
def test_many_rows(dtype, hd, heads_outside, form):
    """Row tiles that begin and end inside a token's heads, and tiles of positions that end inside a page."""
    check(Paged(dtype, [150, 37, 129], [150, 300, 140], 6, 2, hd, 32, heads_outside=heads_outside, tail_rows=3), form)


@pytest.mark.parametrize("dtype,hd,page", [("bf16", 64, 64), ("bf16", 128, 16), ("fp32", 64, 16)])
@pytest.mark.parametrize("causal", [True, False])
def test_one_token_of_a_long_context(dtype, hd, page, causal):
    """One sequence: its context is split over the GPU and the parts are joined."""
    check(Paged(dtype, [1], [5003], 8, 2, hd, page), dict(causal=causal))


def test_few_rows_of_long_contexts_with_a_window():
    check(Paged("bf16", [2, 5], [3001, 2500], 8, 2, 64, 16), dict(window=700))
    check(Paged("bf16", [2, 5], [3001, 2500], 8, 2, 64, 16), dict(window=700), max_kv=188 * 16, max_new=7)


@pytest.mark.parametrize("dtype,hd", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_rows_that_see_nothing(dtype, hd):
    """More new rows than positions: those before the first position see nothing, and are zeros."""
    p = Paged(dtype, [5, 2, 3], [2, 0, 3], 4, 2, hd, 16)
    out = check(p)
    assert bool((out[:3] == 0).all()) and bool((out[5:7] == 0).all())


@pytest.mark.parametrize("dtype,hd,rows", [("fp32", 16, 40), ("bf16", 64, 40), ("bf16", 128, 200), ("bf16", 64, 300)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_a_row_does_not_see_may_hold_anything(dtype, hd, rows, bad):
    """Keys and values of later positions are not numbers: only the rows that see them notice."""
    p = Paged(dtype, [rows], [rows + 100], 4, 2, hd, 16)
    at = rows + 60
    page, slot = int(p.table[0, at // 16]), at % 16
    p.v_pool[page, :, slot, 3] = bad
    p.v[0][at, :, 3] = bad
    clean = list(range(0, rows - 40))
    check(p, rows=clean, lse=False)
    eng = engine(dtype)
    out = eng.paged_attention(p.kv(), p.q.cuda())
    eng.sync()
    assert not bool(torch.isfinite(out[rows - 40:, :, 3].float()).any())
    others = [d for d in range(hd) if d != 3]
    assert bool(torch.isfinite(out[:, :, others].float()).all())
    p.k_pool[page, :, slot, 0] = bad
    check(p, rows=clean, lse=False)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("fp32", 16)])
def test_positions_that_left_the_window_may_hold_anything(dtype, hd):
    p = Paged(dtype, [60, 1], [400, 300], 4, 2, hd, 16)
    for b, upto in ((0, 400 - 60 - 50 + 1), (1, 300 - 50)):
        for t in range(upto):
            p.v_pool[int(p.table[b, t // 16]), :, t % 16] = math.nan
            p.k_pool[int(p.table[b, t // 16]), :, t % 16] = math.inf
    check(p, dict(window=50))


def test_large_scores_and_equal_ones():
    p = Paged("bf16", [3, 130], [700, 260], 4, 2, 64, 16)
    check(p, dict(scale=4.0), lse=False)
    check(p, dict(scale=0.0))
    check(p, dict(scale=-0.2))


@pytest.mark.parametrize("dtype,hd,rows", [("bf16", 64, 1), ("bf16", 128, 130), ("fp32", 16, 3)])
def test_offsets_beyond_32_bits(dtype, hd, rows):
    """A pool of more than 2^32 bytes and 2^31 elements per side: the last pages are used."""
    es = 2 if dtype == "bf16" else 4
    small = Paged(dtype, [rows], [rows + 150], 4, 2, hd, 64)
    per_page = 2 * 64 * hd
    n = (2 ** 31 + 2 ** 28) // per_page
    if n * per_page * es * 2 > 60e9:
        pytest.skip("pool")
    k, v = (torch.empty(n, 2, 64, hd, dtype=small.dt, device="cuda") for _ in range(2))
    used = small.k_pool.shape[0]
    k[n - used:], v[n - used:] = small.k_pool, small.v_pool
    small.k_pool, small.v_pool = k, v
    small.d_table = (small.table + (n - used)).cuda()
    check(small)


def test_strided_rows_and_tables():
    """q as columns of a fused QKV product, out inside wider rows, a page table with room for more."""
    p = Paged("bf16", [3, 40], [100, 77], 4, 2, 64, 16)
    eng = engine("bf16")
    want, _, tol = reference(p)
    qkv = torch.randn(p.rows, 8, 64, dtype=torch.bfloat16, device="cuda")
    qkv[:, :4] = p.q.cuda()
    wide = torch.full((p.rows, 6, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    table = torch.full((2, 50), -5, dtype=torch.int32, device="cuda")
    table[:, : p.d_table.shape[1]] = p.d_table
    p.d_table = table[:, : p.d_table.shape[1] + 2]
    eng.paged_attention(p.kv(), qkv[:, :4], out=wide[:, 1:5])
    eng.sync()
    assert bool(((wide[:, 1:5].double().cpu() - want).abs() <= tol).all())
    assert bool((wide[:, 0] == 3).all()) and bool((wide[:, 5] == 3).all())


def test_pages_shared_by_sequences():
    """Two beams of one user share the pages of the history."""
    p = Paged("bf16", [1, 1], [129, 129], 8, 2, 64, 64)
    p.table[1, :2] = p.table[0, :2]
    p.d_table = p.table.cuda()
    p.k[1][:128], p.v[1][:128] = p.k[0][:128], p.v[0][:128]
    check(p)


@pytest.mark.parametrize("dtype,hd,news,lens", [("bf16", 64, [1], [4000]), ("bf16", 128, [300], [1500]), ("fp32", 16, [2, 3], [300, 70])])
def test_a_captured_call_and_repeats(dtype, hd, news, lens):
    """The same bits from every repeat, from a graph, and with other lengths in the same buffers from the same graph."""
    p = Paged(dtype, news, lens, 8, 2, hd, 16)
    s = torch.cuda.Stream()
    eng = engine(dtype, stream=s)
    q, kv = p.q.cuda(), p.kv()
    torch.cuda.synchronize()
    first = eng.paged_attention(kv, q)
    again = eng.paged_attention(kv, q)
    eng.sync()
    assert torch.equal(first, again)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = eng.paged_attention(kv, q)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    shorter = [max(n, l // 2) for n, l in zip(news, lens)]
    p.kv_len.copy_(torch.tensor(shorter, dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    p.lens = shorter
    p.k, p.v = [k[:n] for k, n in zip(p.k, shorter)], [v[:n] for v, n in zip(p.v, shorter)]
    want, _, tol = reference(p)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())


def test_two_graphs_at_once():
    """Two captured calls on two streams, each with the workspace that its capture gave it."""
    outs, graphs, wants = [], [], []
    keep = []
    for i in range(2):
        p = Paged("bf16", [1], [6000 + 500 * i], 8, 2, 64, 16, seed=i)
        s = torch.cuda.Stream()
        eng = engine("bf16", stream=s)
        q, kv = p.q.cuda(), p.kv()
        torch.cuda.synchronize()
        wants.append(eng.paged_attention(kv, q))
        eng.sync()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(eng.paged_attention(kv, q))
        graphs.append((g, s))
        keep.append((p, q, kv, eng))
    for _ in range(20):
        for g, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for out, want in zip(outs, wants):
        assert torch.equal(out, want)


def bad_call(p, status, **kw):
    from paper_2511_18793_b200 import binding
    eng = engine(p.dtype)
    with pytest.raises(binding.NezhaError) as e:
        eng.paged_attention(p.kv(**{k: kw.pop(k) for k in list(kw) if k.startswith("max_")}), p.q.cuda(), **kw)
        eng.sync()
    assert e.value.status == status
    eng.sync()


def test_refused_calls():
    p = Paged("bf16", [2], [40], 4, 2, 64, 16)
    for kw in (dict(window=-1), dict(window=3, causal=False), dict(softcap=-1.0), dict(softcap=math.nan), dict(scale=math.inf),
               dict(max_kv=p.table.shape[1] * 16 + 1), dict(max_kv=-1)):
        bad_call(p, 1, **kw)
    p.q = torch.randn(2, 3, 64, dtype=torch.bfloat16)          # 3 query heads on 2 KV heads
    bad_call(p, 1)


@pytest.mark.parametrize("dtype,hd,n", [("fp32", 16, 2), ("bf16", 64, 2), ("bf16", 128, 140)])
def test_bad_contents_are_reported(dtype, hd, n):
    """Pages outside the pool, lengths and row ranges beyond the bounds: an error from the next synchronising call, and the other sequence's
    rows as they should be."""
    def make():
        return Paged(dtype, [n, 3], [n + 60, 90], 4, 2, hd, 16)
    eng = engine(dtype)
    from paper_2511_18793_b200 import binding
    good = make()
    want, _, tol = reference(good)
    for what in ("page high", "page low", "length", "negative length", "rows", "descending"):
        p = make()
        kv = p.kv(max_kv=max(p.lens))
        if what == "page high":
            p.d_table[0, 1] = p.k_pool.shape[0]
        elif what == "page low":
            p.d_table[0, 0] = -1
        elif what == "length":
            p.kv_len[0] = max(p.lens) + 1
        elif what == "negative length":
            p.kv_len[0] = -3
        elif what == "rows":
            p.row_start[0] = -2
        else:
            p.row_start[0] = n + 1
        out = torch.zeros(p.rows, 4, hd, dtype=p.dt, device="cuda")
        eng.paged_attention(kv, p.q.cuda(), out=out)
        with pytest.raises(binding.NezhaError) as e:
            eng.sync()
        assert e.value.status == 8, what
        eng.sync()
        if what != "descending":
            assert bool(((out.double().cpu() - want).abs() <= tol)[n:].all()), what
