"""8-bit rows and products: whole numbers, so equal to the definition and not merely near it."""
import math

import pytest
import torch

from paged_helpers import engine

pytestmark = pytest.mark.gpu


def quantized(x):
    """The definition with the exact quotient: 127 x and the maximum are exact in 64 bits, and no quotient of two such numbers is nearer to a
    half than 64 bits resolve unless it is one."""
    x = x.double()
    top = x.abs().max(dim=1).values
    q = torch.round(127.0 * x / torch.where(top > 0, top, torch.ones_like(top))[:, None])
    return q.to(torch.int8), (top / 127.0).float()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (20, 2048), (33, 64), (5, 1000), (17, 4872), (64, 11008), (2, 40000), (9, 20001)])
def test_rows_equal_the_definition(dtype, M, K):
    eng = engine(dtype)
    x = (torch.randn(M, K, generator=torch.Generator().manual_seed(M * K)) * 3).to(eng.dtype)
    x[0, ::5] = x[0].abs().max() / 2                     # halves of the largest: on the border 63.5
    x[0, 1::5] = -x[0].abs().max() / 2
    q, s = eng.quantize_rows(x.cuda())
    eng.sync()
    want_q, want_s = quantized(x)
    assert torch.equal(q.cpu(), want_q) and torch.equal(s.cpu(), (x.float().abs().max(dim=1).values / 127.0))
    assert torch.allclose(s.cpu(), want_s, rtol=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_extremes(dtype):
    eng = engine(dtype)
    rows = torch.zeros(8, 72)
    rows[1] = 1e-38
    rows[2, 3] = 3e38
    rows[3, 5] = math.nan
    rows[4, 6] = -math.inf
    rows[5, :2] = torch.tensor([1e-40, -5e-41])
    rows[6, :3] = torch.tensor([1.0, -0.0, 1e-30])
    rows[7] = torch.linspace(-1, 1, 72)
    x = rows.to(eng.dtype)
    q, s = eng.quantize_rows(x.cuda())
    eng.sync()
    q, s = q.cpu(), s.cpu()
    good = [0, 1, 2, 5, 6, 7]
    want_q, _ = quantized(x[good])
    assert torch.equal(q[good], want_q)
    assert bool((q[3:5] == 0).all()) and bool(torch.isnan(s[3:5]).all())
    assert s[0] == 0


def test_strided_rows_and_rows_behind():
    eng = engine("bf16")
    wide = torch.randn(10, 640, device="cuda").bfloat16()
    for x in (wide[:, 64:320], wide[:, 3:130], wide[1:4, :512]):
        q = torch.full((x.shape[0] + 1, x.shape[1]), 99, dtype=torch.int8, device="cuda")
        s = torch.full((x.shape[0] + 1,), 7.0, device="cuda")
        eng.quantize_rows(x, q[:-1], s[:-1])
        eng.sync()
        want_q, _ = quantized(x.cpu())
        assert torch.equal(q[:-1].cpu(), want_q) and bool((q[-1] == 99).all()) and s[-1] == 7.0


def product(a, sa, w, sw, bias=None):
    """The kernels' roundings after the exact sum: to fp32, two products, a sum."""
    acc = (a.double().cuda() @ w.double().cuda().T).cpu()
    x = acc.float() * sa[:, None] * sw[None, :]
    return x if bias is None else x + bias


def operands(M, N, K, seed=0, extreme=False):
    g = torch.Generator().manual_seed(seed + M + N + K)
    a, w = (torch.randint(-128, 128, (n, K), generator=g).to(torch.int8) for n in (M, N))
    if extreme:
        a[:], w[:] = -128, -128
    return a, torch.rand(M, generator=g) + 0.1, w, torch.rand(N, generator=g) * 1e-3 + 1e-4, torch.randn(N, generator=g)


SIZES = [(1, 1, 1), (1, 32, 64), (3, 5, 7), (1, 2048, 2048), (20, 1056, 512), (33, 64, 1024), (48, 100, 128), (64, 4096, 896), (65, 129, 96), (100, 250, 48),
         (128, 512, 4864), (129, 256, 128), (200, 1000, 1008), (257, 300, 2048), (384, 9728, 896), (640, 1536, 8960), (970, 4864, 896), (1000, 77, 64), (2049, 2048, 512)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("with_bias", [False, True])
def test_products_equal_the_definition(M, N, K, with_bias):
    eng = engine("bf16")
    a, sa, w, sw, bias = operands(M, N, K)
    bias = bias if with_bias else None
    dev = [t.cuda() for t in (a, sa, w, sw)]
    want = product(a, sa, w, sw, bias)
    room = torch.full((M + 1, N), 3.0, device="cuda")
    for epilogue in (1, 0, 2):
        dt = torch.bfloat16 if epilogue == 0 else torch.float32
        room = torch.full((M + 1, N), 3.0, device="cuda", dtype=dt)
        eng.gemm_int8(*dev, room[:M], epilogue=epilogue, bias=None if bias is None else bias.cuda())
        eng.sync()
        got = room[:M].cpu()
        ref = want if epilogue == 1 else want.bfloat16() if epilogue == 0 else torch.full((M, N), 3.0) + want
        assert torch.equal(got, ref), (epilogue, float((got.float() - ref.float()).abs().max()))
        assert bool((room[M] == 3.0).all())


@pytest.mark.parametrize("M", [1, 40, 200])
def test_the_largest_sums_fit(M):
    """Every operand at its most negative and the longest K: the sum is one step short of 2^31."""
    eng = engine("bf16")
    for K in (131071, 131056):
        a, sa, w, sw, _ = operands(M, 64, K, extreme=True)
        out = torch.empty(M, 64, device="cuda")
        eng.gemm_int8(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), out, epilogue=1)
        eng.sync()
        assert torch.equal(out.cpu(), torch.full((M, 64), float(K * 16384)) * sa[:, None] * sw[None])


@pytest.mark.parametrize("M,N,K", [(20, 64, 256), (300, 96, 512)])
def test_misaligned_operands_and_fp32_engines(M, N, K):
    eng = engine("fp32")
    a, sa, w, sw, bias = operands(M, N, K)
    room = torch.empty(M * K + 1, dtype=torch.int8, device="cuda")
    room[1:] = a.cuda().flatten()
    want = product(a, sa, w, sw, bias)
    for A in (a.cuda(), room[1:].view(M, K)):
        out = torch.empty(M, N, device="cuda")
        eng.gemm_int8(A, sa.cuda(), w.cuda(), sw.cuda(), out, epilogue=0, bias=bias.cuda())
        eng.sync()
        assert torch.equal(out.cpu(), want)
    for off in (1, 2, 3):                                  # C at any element
        cbuf = torch.empty(M * N + 4, device="cuda")
        out = cbuf[off: off + M * N].view(M, N)
        eng.gemm_int8(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), out, epilogue=1, bias=bias.cuda())
        eng.sync()
        assert torch.equal(out.cpu(), want)


def test_bf16_result_at_any_element():
    eng = engine("bf16")
    a, sa, w, sw, _ = operands(50, 64, 256)
    for off in (1, 2, 4):
        cbuf = torch.empty(50 * 64 + 4, device="cuda", dtype=torch.bfloat16)
        out = cbuf[off: off + 50 * 64].view(50, 64)
        eng.gemm_int8(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), out)
        eng.sync()
        assert torch.equal(out.cpu(), product(a, sa, w, sw).bfloat16())


def test_a_quantized_row_that_is_not_a_number_gives_nan():
    eng = engine("bf16")
    x = torch.randn(4, 256, device="cuda").bfloat16()
    x[2, 9] = math.inf
    w = torch.randn(64, 256, device="cuda").bfloat16()
    qx, sx = eng.quantize_rows(x)
    qw, sw = eng.quantize_rows(w)
    out = eng.gemm_int8(qx, sx, qw, sw, torch.empty(4, 64, device="cuda"), epilogue=1)
    eng.sync()
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isfinite(out[[0, 1, 3]]).all())


def test_a_captured_product():
    s = torch.cuda.Stream()
    eng = engine("bf16", stream=s)
    for M, N, K in ((20, 4096, 2048), (300, 2048, 512)):
        a, sa, w, sw, _ = [t.cuda() for t in operands(M, N, K)]
        torch.cuda.synchronize()
        want = eng.gemm_int8(a, sa, w, sw, torch.empty(M, N, device="cuda", dtype=torch.bfloat16))
        eng.sync()
        out = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            eng.gemm_int8(a, sa, w, sw, out)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refused_calls():
    from paper_2511_18793_b200 import binding
    eng = engine("bf16")
    a, sa, w, sw, _ = [t.cuda() for t in operands(4, 32, 64)]
    out = torch.empty(4, 32, device="cuda")
    lib, h = binding.lib, eng._h
    def call(A=a.data_ptr(), M=4, N=32, K=64, epilogue=1):
        return lib.nezha_gemm_int8(h, A, sa.data_ptr(), w.data_ptr(), sw.data_ptr(), out.data_ptr(), M, N, K, epilogue, None)
    assert call(A=None) == 1 and call(M=0) == 1 and call(K=0) == 1 and call(epilogue=3) == 1 and call(K=131072) == 7
    assert lib.nezha_gemm_int8(h, a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), out.data_ptr() + 2, 4, 32, 64, 1, None) == 1
    x = torch.randn(4, 64, device="cuda").bfloat16()
    q, s = torch.empty(4, 64, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    assert lib.nezha_quantize_rows(h, x.data_ptr(), 63, 4, 64, q.data_ptr(), s.data_ptr()) == 1
    assert lib.nezha_quantize_rows(h, None, 64, 4, 64, q.data_ptr(), s.data_ptr()) == 1
    assert lib.nezha_quantize_rows(h, x.data_ptr(), 64, 0, 64, q.data_ptr(), s.data_ptr()) == 0
