"""Which kernel serves a call: a call that ran on the way down (a tensor map refused, registers that do not add up) would be right all the same."""
import json

import pytest
import torch
from torch.profiler import ProfilerActivity, profile

from paged_helpers import Paged, engine

pytestmark = pytest.mark.gpu


def launched(call, path):
    """The names of the library's kernels that the call launches."""
    call()                                               # (one-time set-up)
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as p:
        torch.zeros(1, device="cuda")
        call()
        torch.cuda.synchronize()
    p.export_chrome_trace(str(path))
    names = [e["name"] for e in json.loads(path.read_text())["traceEvents"] if e.get("cat") == "kernel"]
    if not names:
        pytest.skip("no activity records: another profiler holds the process")
    return [n.split("(anonymous namespace)::")[1].split(">(")[0] + ">" for n in names if "nz::(anonymous namespace)::" in n]


#: (type, head dimension, new rows of each sequence, form, page size) -> the kernel that attends
ATTENTION = [
    ("fp32", 16, [3], {}, 16, "paged_attn_simt_kernel<float, 16>"), ("bf16", 32, [300], {}, 16, "paged_attn_simt_kernel<__nv_bfloat16, 32>"),
    ("bf16", 64, [8], {}, 16, "paged_attn_token_kernel<64, 4, false, true>"), ("bf16", 128, [1], dict(softcap=9.0), 16, "paged_attn_token_kernel<128, 2, true, true>"),
    ("bf16", 64, [9], {}, 16, "paged_attn_tc_kernel<64, 1, 2, false, true>"), ("bf16", 128, [17], {}, 8, "paged_attn_tc_kernel<128, 4, 1, false, true>"),
    ("bf16", 64, [200], {}, 20, "paged_attn_tc_kernel<64, 4, 1, false, false>"),
    ("bf16", 64, [70], dict(softcap=1e30), 16, "paged_attn_tc_kernel<64, 4, 1, true, true>"),      # a cap that the series does not bear
]
# the tcgen05 kernel in all its forms: one, two and four tiles of 128 rows a CTA
ATTENTION += [("bf16", hd, news, form, page, f"paged_attn_umma_kernel<{hd}, {n}, {nx}>")
              for hd, nx, news, page in ((64, 1, [65], 16), (64, 2, [129], 64), (64, 4, [300] + [270] * 99, 16), (128, 1, [128], 24), (128, 2, [300] + [270] * 99, 32))
              for n, form in enumerate(({}, dict(softcap=9.0), dict(slopes=True), dict(softcap=30.0, slopes=True)))]


@pytest.mark.parametrize("dtype,hd,news,form,page,kernel", ATTENTION, ids=[c[-1] for c in ATTENTION])
def test_attention(dtype, hd, news, form, page, kernel, tmp_path):
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = torch.full((1,), 0.1, device="cuda")
    p = Paged(dtype, news, [n + 20 for n in news], 1, 1, hd, page)
    eng, kv, q = engine(dtype), p.kv(), p.q.cuda()
    got = launched(lambda: eng.paged_attention(kv, q, **form), tmp_path / "trace.json")
    eng.sync()
    assert [n for n in got if "join" not in n] == [kernel], got


@pytest.mark.parametrize("M,N,K,epilogue,kernel", [
    (20, 2048, 2048, 0, "gemm_i8_skinny_kernel<32, 0>"), (33, 1024, 2048, 1, "gemm_i8_skinny_kernel<64, 1>"), (100, 1024, 2048, 2, "gemm_i8_skinny_kernel<128, 2>"),
    (971, 9728, 896, 1, "gemm_i8_kernel<192, 1>"), (8192, 4096, 2048, 0, "gemm_i8_pair_kernel<0>"), (300, 64, 40, 0, "gemm_i8_simt_kernel<__nv_bfloat16, false>")])
def test_products(M, N, K, epilogue, kernel, tmp_path):
    eng = engine("bf16")
    a, w = (torch.ones(n, K, dtype=torch.int8, device="cuda") for n in (M, N))
    sa, sw = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    out = torch.zeros(M, N, dtype=torch.float32 if epilogue else torch.bfloat16, device="cuda")
    got = launched(lambda: eng.gemm_int8(a, sa, w, sw, out, epilogue=epilogue), tmp_path / "trace.json")
    eng.sync()
    assert got == [kernel], got


@pytest.mark.parametrize("dtype,M,K,kernel", [
    ("bf16", 20, 2048, "quantize_rows_kernel<__nv_bfloat16, 128, true>"), ("fp32", 7, 33, "quantize_rows_kernel<float, 32, false>"),
    ("bf16", 16008, 1024, "quantize_stream_kernel<__nv_bfloat16, 32>"), ("fp32", 2000, 11008, "quantize_stream_kernel<float, 512>")])
def test_rows_to_8_bits(dtype, M, K, kernel, tmp_path):
    eng = engine(dtype)
    x = torch.ones(M, K, dtype=eng.dtype, device="cuda")
    got = launched(lambda: eng.quantize_rows(x), tmp_path / "trace.json")
    eng.sync()
    assert got == [kernel], got
