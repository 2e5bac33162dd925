"""Contexts that end next to 2^31 positions: a table that repeats one large page describes them, a window keeps the work small."""
import math
from types import SimpleNamespace

import pytest
import torch

from paged_helpers import TYPES, engine, reference

pytestmark = pytest.mark.gpu

PAGE, PAGES, MOST = 2 ** 20, 2048, 2 ** 31 - 4096


def far(dtype, hd, new, window, hq=2, seed=0):
    """`new` rows at the end of MOST positions.  `near` holds what they see, shifted so that its last position is the context's last."""
    g = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype]
    seen = window + new
    k, v = (torch.randn(seen, 1, hd, generator=g).to(dt) for _ in range(2))
    pool_k, pool_v = (torch.full((1, 1, PAGE, hd), math.nan, dtype=dt, device="cuda") for _ in range(2))
    slots = (torch.arange(MOST - seen, MOST) % PAGE).cuda()
    pool_k[0, 0, slots], pool_v[0, 0, slots] = k[:, 0].cuda(), v[:, 0].cuda()
    q = torch.randn(new, hq, hd, generator=g).to(dt)
    near = SimpleNamespace(dtype=dtype, news=[new], lens=[seen], hq=hq, hkv=1, hd=hd, rows=new, starts=[0, new], q=q, k=[k], v=[v])
    table = torch.zeros(1, PAGES, dtype=torch.int32, device="cuda")
    start, length = torch.tensor([0, new], dtype=torch.int32).cuda(), torch.tensor([MOST], dtype=torch.int32).cuda()
    torch.cuda.synchronize()
    return near, (pool_k, pool_v, table, start, length, new, MOST)


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("fp32", 64), ("bf16", 32), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("new", [1, 6, 30, 150])
@pytest.mark.parametrize("window", [70, 300, 1500])
def test_the_last_positions(dtype, hd, new, window):
    from paper_2511_18793_b200 import binding
    near, args = far(dtype, hd, new, window)
    eng = engine(dtype)
    lse = torch.empty(new, 2, device="cuda")
    out = eng.paged_attention(binding.PagedKV(*args), near.q.cuda(), window=window, lse=lse)
    eng.sync()
    rows = sorted({0, new // 2, new - 1})
    want, want_lse, tol = reference(near, window=window, rows=rows)
    assert bool(((out.double().cpu() - want).abs() <= tol)[rows].all())
    assert bool(((lse.double().cpu() - want_lse).abs()[rows] <= 2e-5 * (1 + want_lse.abs()[rows])).all())


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64)])
def test_an_append_at_the_last_positions(dtype, hd):
    from paper_2511_18793_b200 import binding
    near, args = far(dtype, hd, 5, 10)
    x = torch.randn(5, 2, hd, device="cuda").to(TYPES[dtype])
    eng = engine(dtype)
    eng.kv_append(binding.PagedKV(*args), x[:, :1], x[:, 1:])
    eng.sync()
    slots = (torch.arange(MOST - 5, MOST) % PAGE).cuda()
    for pool, src in ((args[0], x[:, 0]), (args[1], x[:, 1])):
        assert torch.equal(pool[0, 0, slots], src)
        assert bool(torch.isnan(pool[0, 0, (slots + 5) % PAGE]).all())
