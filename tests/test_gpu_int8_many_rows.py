"""Rows to 8 bits where there are many (a ring of rows in shared memory): equal to the definition, computed in 64 bits on the device."""
import math

import pytest
import torch

from paged_helpers import engine
from test_gpu_int8 import quantized

pytestmark = pytest.mark.gpu


# each number of threads per row, the longest rows that have room and one that has not, the last row tile full and not
@pytest.mark.parametrize("dtype,M,K", [("bf16", 33001, 504), ("bf16", 10001, 1608), ("bf16", 8192, 2048), ("bf16", 2600, 6400), ("bf16", 1301, 12808),
                                       ("bf16", 640, 25608), ("bf16", 333, 51200), ("bf16", 330, 51208), ("fp32", 17003, 500), ("fp32", 2001, 4100),
                                       ("fp32", 700, 25596)])
def test_many_rows_equal_the_definition(dtype, M, K):
    eng = engine(dtype)
    g = torch.Generator(device="cuda").manual_seed(M + K)
    x = (torch.randn(M, K, generator=g, device="cuda") * 3).to(eng.dtype)
    x[1, ::5] = x[1].abs().max() / 2                     # halves of the largest: on the border 63.5
    x[M - 1] = 0
    x[M // 2, K - 1] = math.nan
    q = torch.full((M + 1, K), 99, dtype=torch.int8, device="cuda")
    s = torch.full((M + 1,), 7.0, device="cuda")
    torch.cuda.synchronize()
    eng.quantize_rows(x, q[:-1], s[:-1])
    eng.sync()
    good = torch.ones(M, dtype=torch.bool, device="cuda")
    good[M // 2] = False
    for at in range(0, M, 4096):                         # (the definition takes a few times the room of its rows)
        part = slice(at, min(M, at + 4096))
        want_q, _ = quantized(x[part][good[part]])
        assert torch.equal(q[:-1][part][good[part]], want_q)
        # (on the CPU: a division by a number is a product with its inverse in this library's CUDA code)
        assert torch.equal(s[:-1][part][good[part]].cpu(), x[part][good[part]].float().abs().max(dim=1).values.cpu() / 127.0)
    assert bool((q[M // 2] == 0).all()) and bool(torch.isnan(s[M // 2]))
    assert bool((q[M] == 99).all()) and s[M] == 7.0


def test_many_strided_rows():
    eng = engine("bf16")
    wide = torch.randn(9000, 4160, device="cuda").bfloat16()
    for x in (wide[:, 64:2112], wide[:, 3:2051]):        # in 16-byte pieces, and not
        torch.cuda.synchronize()
        q, s = eng.quantize_rows(x)
        eng.sync()
        want_q, _ = quantized(x)
        assert torch.equal(q, want_q)


def test_captured_many_rows():
    """The same bits from a graph, next to another stream's call."""
    s = torch.cuda.Stream()
    eng, other = engine("bf16", stream=s), engine("bf16")
    x = torch.randn(9000, 2048, device="cuda").bfloat16()
    y = torch.randn(9000, 2048, device="cuda").bfloat16()
    q, sc = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(9000, device="cuda")
    torch.cuda.synchronize()
    eng.quantize_rows(x, q, sc)
    eng.sync()
    want, want_s = q.clone(), sc.clone()
    q.zero_()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        eng.quantize_rows(x, q, sc)
    for _ in range(5):
        with torch.cuda.stream(s):
            g.replay()
        qy, sy = other.quantize_rows(y)
    torch.cuda.synchronize()
    assert torch.equal(q, want) and torch.equal(sc, want_s)
    assert torch.equal(qy, quantized(y)[0])
