"""Sequences that share rows of the page table."""
import pytest
import torch

from paged_helpers import Paged
from test_gpu_paged_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd,new", [("fp32", 16, 2), ("bf16", 64, 1), ("bf16", 128, 12), ("bf16", 64, 90)])
def test_one_table_row_for_all_sequences(dtype, hd, new):
    """The beams of one user, on the pages of one history: the table is expanded, not copied."""
    p = Paged(dtype, [new] * 4, [new + 150] * 4, 4, 2, hd, 16)
    for b in range(1, 4):
        p.k[b], p.v[b] = p.k[0], p.v[0]
    one = p.d_table[:1]
    rows = sorted({0, new - 1, new, 2 * new, 4 * new - 1})
    for b, n in ((1, 40), (3, 99)):                  # of different lengths
        p.lens[b], p.k[b], p.v[b] = new + n, p.k[0][: new + n], p.v[0][: new + n]
    p.kv_len = torch.tensor(p.lens, dtype=torch.int32).cuda()
    p.d_table = one.expand(4, -1)
    check(p, rows=rows)


def test_tables_that_overlap():
    """Sequence b has the pages from the b-th of a list on."""
    p = Paged("bf16", [1, 1, 1], [64, 64, 64], 4, 2, 64, 16)
    every = torch.cat([p.d_table[0], p.d_table[1, :2]])
    k, v = torch.cat([p.k[0], p.k[1][:32]]), torch.cat([p.v[0], p.v[1][:32]])
    for b in range(3):
        p.k[b], p.v[b] = k[16 * b: 16 * b + 64], v[16 * b: 16 * b + 64]
    p.d_table = every.as_strided((3, 4), (1, 1))
    check(p)
