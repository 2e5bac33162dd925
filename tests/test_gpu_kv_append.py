"""Rotary positions and the append to a paged cache against the formula in 64 bits."""
import math

import pytest
import torch

from paged_helpers import HALF, Paged, engine

pytestmark = pytest.mark.gpu


def frequencies(rope):
    r = rope.rot_dim
    out, mag = [], rope.magnitude or 1.0
    theta = float(torch.tensor(rope.theta, dtype=torch.float32))
    for i in range(r // 2):
        f = theta ** (-2.0 * i / r)
        if rope.scaling == "linear":
            f /= rope.factor
        if rope.scaling == "parts":
            fast, slow = (rope.turns_fast, rope.turns_slow) if rope.turns_fast else (32.0, 1.0)
            pair = [r * math.log(rope.trained_positions / (n * 2 * math.pi)) / (2 * math.log(theta)) for n in (fast, slow)]
            lo, hi = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), r - 1)
            g = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = f * (1 - g) + f / rope.factor * g
            mag = rope.magnitude or 0.1 * math.log(rope.factor) + 1.0
        out.append(f)
    return torch.tensor(out, dtype=torch.float64), mag


def turned(x, pos, rope):
    """(rotated x, the sizes that its roundings go by); x [rows, heads, hd] in 64 bits."""
    f, mag = frequencies(rope)
    ang = pos.double()[:, None] * f
    c, s = (torch.cos(ang) * mag)[:, None], (torch.sin(ang) * mag)[:, None]
    r = rope.rot_dim
    ia = torch.arange(0, r, 2) if rope.interleaved else torch.arange(r // 2)
    ib = ia + 1 if rope.interleaved else ia + r // 2
    y, size = x.clone(), torch.zeros_like(x)
    y[..., ia], y[..., ib] = x[..., ia] * c - x[..., ib] * s, x[..., ib] * c + x[..., ia] * s
    both = (x[..., ia].abs() + x[..., ib].abs()) * mag
    size[..., ia], size[..., ib] = both, both
    return y, size


def check(p, rope, positions=None, in_place=False, with_q=True, n_table=None, fused=True, eng=None):
    eng = eng or engine(p.dtype)
    g = torch.Generator().manual_seed(5)
    heads = p.hq + 2 * p.hkv
    x = torch.randn(p.rows, heads, p.hd, generator=g).to(p.dt)
    pos = torch.cat([torch.arange(l - n, l) for n, l in zip(p.news, p.lens)] + [torch.zeros(p.rows - p.starts[-1], dtype=torch.long)])
    turn = pos if positions is None else positions
    xd = x.cuda()
    q, k, v = xd[:, : p.hq], xd[:, p.hq: p.hq + p.hkv], xd[:, p.hq + p.hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    k_before, v_before = p.k_pool.clone(), p.v_pool.clone()
    q_out = None
    if with_q:
        q_out = q if in_place else torch.full((p.rows, p.hq, p.hd), 9.0, dtype=p.dt, device="cuda")
    tab = None if rope is None else eng.rope_table(rope, int(turn.max()) + 1 if n_table is None else n_table)
    got = eng.kv_append(p.kv(), k, v, q=q if with_q else None, rope=tab, q_out=q_out,
                        positions=None if positions is None else positions.to(torch.int32).cuda())
    eng.sync()
    xf = x.double()
    if rope is None:
        want_q, want_k = xf[:, : p.hq], xf[:, p.hq: p.hq + p.hkv]
        size_q, size_k = torch.zeros_like(want_q), torch.zeros_like(want_k)
    else:
        want_q, size_q = turned(xf[:, : p.hq], turn, rope)
        want_k, size_k = turned(xf[:, p.hq: p.hq + p.hkv], turn, rope)
    # cosine, sine, two products and a sum in 32 bits, then the storage type's rounding
    n = p.starts[-1]
    if with_q:
        err, tol = (got.double().cpu() - want_q).abs(), HALF[p.dtype] * want_q.abs() + 4 * 2.0 ** -24 * size_q
        assert bool((err <= tol)[:n].all()), float((err - tol)[:n].max())
        if not in_place:
            assert bool((got[n:] == 9.0).all())
    want_kp, want_vp = k_before.double().cpu(), v_before.cpu()
    tol_kp = torch.zeros_like(want_kp)
    for b in range(len(p.news)):
        for i in range(p.news[b]):
            row, t = p.starts[b] + i, p.lens[b] - p.news[b] + i
            page, slot = int(p.table[b, t // p.page]), t % p.page
            want_kp[page, :, slot] = want_k[row]
            tol_kp[page, :, slot] = HALF[p.dtype] * want_k[row].abs() + 4 * 2.0 ** -24 * size_k[row]
            want_vp[page, :, slot] = x[row, p.hq + p.hkv:]
    assert torch.equal(p.v_pool.cpu(), want_vp)
    assert bool(((p.k_pool.double().cpu() - want_kp).abs() <= tol_kp).all())


NEWS, LENS = [1, 0, 3, 17, 1, 2], [1, 5, 3, 90, 129, 64]


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("fp32", 4, 4, 16), ("fp32", 3, 1, 128), ("bf16", 4, 2, 16), ("bf16", 4, 4, 32), ("bf16", 14, 2, 64), ("bf16", 12, 2, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("part", [1.0, 0.5, "odd"])
def test_layouts_and_parts(dtype, hq, hkv, hd, interleaved, part):
    from paper_2511_18793_b200 import binding
    rot = hd // 2 - 2 if part == "odd" else int(hd * part)
    check(Paged(dtype, NEWS, LENS, hq, hkv, hd, 16, garbage=1.5, tail_rows=2), binding.Rope(rot, interleaved=interleaved))


@pytest.mark.parametrize("page,heads_outside", [(1, True), (5, False), (64, True), (128, False)])
@pytest.mark.parametrize("fused", [True, False])
def test_pages_and_strides(page, heads_outside, fused):
    from paper_2511_18793_b200 import binding
    check(Paged("bf16", NEWS, LENS, 8, 2, 64, page, heads_outside=heads_outside, garbage=-2.0), binding.Rope(64), fused=fused)


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=8.0), dict(scaling="parts", factor=4.0, trained_positions=4096),
                                     dict(scaling="parts", factor=2.0, trained_positions=256, turns_fast=8.0, turns_slow=0.5, magnitude=1.25),
                                     dict(theta=500000.0, magnitude=0.5)])
def test_scalings_and_far_positions(scaling):
    from paper_2511_18793_b200 import binding
    p = Paged("fp32", [5, 2], [70, 40], 4, 2, 64, 16, garbage=0.25)
    far = torch.tensor([0, 1, 999_983, 65_537, 300_001, 7, 1_000_000])
    check(p, binding.Rope(64, **scaling), positions=far)


def test_many_rows_in_place_and_without_queries():
    from paper_2511_18793_b200 import binding
    rope = binding.Rope(128)
    news, lens = [1500, 1200], [1500, 1900]
    check(Paged("bf16", news, lens, 4, 2, 128, 64, garbage=1.0, tail_rows=5), rope)
    check(Paged("bf16", news, lens, 4, 2, 128, 64, garbage=1.0), rope, in_place=True)
    check(Paged("bf16", [30, 1], [30, 64], 4, 2, 128, 64, garbage=1.0), rope, with_q=False)
    check(Paged("bf16", [30, 1], [30, 64], 4, 2, 128, 64, garbage=1.0), None)
    check(Paged("bf16", [3] * 70, [3 + i for i in range(70)], 40, 40, 64, 16, garbage=1.0), binding.Rope(64, interleaved=True))   # more chunks than threads


def test_nan_and_infinities_pass_through():
    """Values that are not rotated arrive bit for bit."""
    eng = engine("bf16")
    p = Paged("bf16", [4], [10], 2, 2, 64, 16, garbage=0.0)
    x = torch.full((4, 6, 64), math.nan, dtype=torch.bfloat16, device="cuda")
    x[1], x[2] = math.inf, -0.0
    eng.kv_append(p.kv(), x[:, 2:4], x[:, 4:])
    eng.sync()
    page = int(p.table[0, 0])
    for pool, src in ((p.k_pool, x[:, 2:4]), (p.v_pool, x[:, 4:])):
        assert torch.equal(pool[page, :, 6:10].transpose(0, 1).contiguous().view(torch.int16), src.contiguous().view(torch.int16))


def test_a_captured_append():
    from paper_2511_18793_b200 import binding
    s = torch.cuda.Stream()
    eng = engine("bf16", stream=s)
    p = Paged("bf16", [2, 3], [40, 50], 4, 2, 64, 16, garbage=0.0)
    x = torch.randn(5, 8, 64, device="cuda").bfloat16()
    tab = eng.rope_table(binding.Rope(64), 64)
    kv = p.kv()
    torch.cuda.synchronize()
    want = eng.kv_append(kv, x[:, 4:6], x[:, 6:], q=x[:, :4], rope=tab)
    eng.sync()
    k_want, v_want = p.k_pool.clone(), p.v_pool.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = eng.kv_append(kv, x[:, 4:6], x[:, 6:], q=x[:, :4], rope=tab)
    p.k_pool.zero_(), p.v_pool.zero_()
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    for b, (n, l) in enumerate(zip(p.news, p.lens)):
        for t in range(l - n, l):
            page = int(p.table[b, t // 16])
            assert torch.equal(p.k_pool[page, :, t % 16], k_want[page, :, t % 16]) and torch.equal(p.v_pool[page, :, t % 16], v_want[page, :, t % 16])


def test_refused_calls():
    from paper_2511_18793_b200 import binding
    eng = engine("bf16")
    p = Paged("bf16", [2], [40], 4, 2, 64, 16, garbage=0.0)
    x = torch.randn(2, 8, 64, device="cuda").bfloat16()
    k, v, q = x[:, 4:6], x[:, 6:], x[:, :4]
    for rope in (dict(rot_dim=63), dict(rot_dim=0), dict(rot_dim=64, theta=1.0), dict(rot_dim=64, scaling="linear", factor=0.5),
                 dict(rot_dim=64, scaling="parts", factor=2.0), dict(rot_dim=64, magnitude=-1.0),
                 dict(rot_dim=64, scaling="parts", factor=2.0, trained_positions=8, turns_fast=1.0, turns_slow=2.0)):
        with pytest.raises(binding.NezhaError) as e:
            eng.rope_table(binding.Rope(**rope), 8)
        assert e.value.status == 1
    wide = eng.rope_table(binding.Rope(128), 64)
    with pytest.raises(binding.NezhaError) as e:                            # more rotated dimensions than the head has
        eng.kv_append(p.kv(), k, v, q=q, rope=wide)
    assert e.value.status == 1
    odd = torch.randn(2 * 8 * 64 + 8, device="cuda").bfloat16()[1: 1 + 2 * 2 * 64].view(2, 2, 64)      # 2 bytes off
    with pytest.raises(binding.NezhaError) as e:
        eng.kv_append(p.kv(), odd, v)
    assert e.value.status == 1 and "16 bytes" in str(e.value)
    overlap = p.k_pool.as_strided(p.k_pool.shape, (64, 64, 64, 1))
    p.k_pool = p.v_pool = overlap
    with pytest.raises(binding.NezhaError) as e:
        eng.kv_append(p.kv(), k, v)
    assert e.value.status == 1


@pytest.mark.parametrize("what", ["page", "table end", "length", "rows", "more rows than positions", "angle"])
def test_bad_contents_are_reported_and_not_written(what):
    from paper_2511_18793_b200 import binding
    eng = engine("bf16")
    p = Paged("bf16", [2, 3], [40, 50], 4, 2, 64, 16, garbage=0.0)
    x = torch.randn(5, 8, 64, device="cuda").bfloat16()
    kv = p.kv(max_kv=50)
    n_table = 64
    if what == "page":
        p.d_table[0, 2] = p.k_pool.shape[0]
    elif what == "table end":
        p.d_table[0, 2] = -1
    elif what == "length":
        p.kv_len[0] = 51
    elif what == "rows":
        p.row_start[2] = 6
    elif what == "more rows than positions":
        p.kv_len[0] = 1
    else:
        n_table = 49
    before_k, before_v = p.k_pool.clone(), p.v_pool.clone()
    tab = eng.rope_table(binding.Rope(64), n_table)
    out = torch.full((5, 4, 64), 2.0, device="cuda", dtype=torch.bfloat16)
    eng.kv_append(kv, x[:, 4:6], x[:, 6:], q=x[:, :4], rope=tab, q_out=out)
    with pytest.raises(binding.NezhaError) as e:
        eng.sync()
    assert e.value.status == 8
    eng.sync()
    bad = {"page": [0, 1], "table end": [0, 1], "length": [0, 1], "rows": [2, 3, 4], "more rows than positions": [0], "angle": [4]}[what]
    for row in range(5):
        assert bool((out[row] == 2.0).all()) == (row in bad), row
    if what in ("page", "table end", "length"):
        for t in (38, 39):
            page = int(p.table[0, t // 16])
            assert torch.equal(p.k_pool[page, :, t % 16], before_k[page, :, t % 16]) and torch.equal(p.v_pool[page, :, t % 16], before_v[page, :, t % 16])
