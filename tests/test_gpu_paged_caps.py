"""Capped scores over the range of caps and scales that is served: what matters is the score, not the sizes of its factors."""
import pytest
import torch

from paged_helpers import Paged
from test_gpu_paged_attention import bad_call, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("fp32", 32)])
@pytest.mark.parametrize("new", [1, 4, 14, 40, 140])
@pytest.mark.parametrize("size,softcap", [(1e10, 1e30), (1e6, 1e30), (1e6, 20.0), (1e7, 20.0), (1e6, 3.0), (1e4, 50.0), (1e3, 1e9), (1e-3, 20.0), (1e-2, 4.0), (1.0, 1e5)])
def test_large_and_small_factors(dtype, hd, new, size, softcap):
    """Queries and keys are `size` times as large as usual and the scale makes up for it."""
    p = Paged(dtype, [new], [new + 150], 4, 1, hd, 16)
    p.q = (p.q.float() * size).to(p.dt)
    for pool, seqs in ((p.k_pool, p.k),):
        pool.copy_((pool.float() * size).to(p.dt))
        seqs[0] = (seqs[0].float() * size).to(p.dt)
    torch.cuda.synchronize()
    check(p, dict(softcap=softcap, scale=hd ** -0.5 / size / size), rows=sorted({0, new // 3, new - 1}))


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("fp32", 32)])
@pytest.mark.parametrize("new", [1, 14, 40])
def test_no_scale_and_the_smallest_caps(dtype, hd, new):
    p = Paged(dtype, [new], [new + 70], 4, 1, hd, 16)
    for form in (dict(softcap=5.0, scale=0.0), dict(softcap=1e-30, scale=0.0), dict(softcap=1e-30, scale=1e-25), dict(softcap=1e-30, scale=-1e-30)):
        check(p, form, rows=sorted({0, new // 3, new - 1}))
    for form in (dict(softcap=9e-31, scale=0.0), dict(softcap=1e-38, scale=1e-40), dict(softcap=1e-44, scale=0.0)):
        bad_call(p, 1, **form)
