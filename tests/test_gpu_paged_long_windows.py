"""Windows next to the largest, and rows far in front of their sequence's first position."""
import pytest
import torch

from paged_helpers import Paged, engine, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64)])
@pytest.mark.parametrize("window", [2 ** 31 - 4097, 2 ** 31 - 8000])
def test_rows_far_in_front_of_the_first_position(dtype, hd, window):
    """6,000 new rows on 50 positions: the first see nothing, and no entry of the table behind the first page is read."""
    from paper_2511_18793_b200 import binding
    new, length, page = 6000, 50, 2 ** 20
    p = Paged(dtype, [new], [length], 1, 1, hd, 64)
    pool_k, pool_v = (torch.zeros(1, 1, page, hd, dtype=p.dt, device="cuda") for _ in range(2))
    pool_k[0, 0, :length], pool_v[0, 0, :length] = p.k[0][:, 0].cuda(), p.v[0][:, 0].cuda()
    table = torch.full((1, 2048), -5, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    eng = engine(dtype)
    out = eng.paged_attention(binding.PagedKV(pool_k, pool_v, table, p.row_start, p.kv_len, new, 2 ** 31 - 4096), p.q.cuda(), window=window)
    eng.sync()
    rows = [0, 900, 1900, 1999, 2000, 5949, 5950, 5951, 5980, 5999]
    want, _, tol = reference(p, window=window, rows=rows)
    assert bool(((out.double().cpu() - want).abs() <= tol)[rows].all())
    assert bool((out[: new - length] == 0).all())
