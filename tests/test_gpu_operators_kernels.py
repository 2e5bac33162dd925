"""Which kernel serves a call: a call that ran on the way down (a tensor map refused, registers that do not add up) would be right all the same."""
import json
import os
import subprocess
import sys
import tempfile

import pytest
import torch
from torch.profiler import ProfilerActivity, profile

pytestmark = pytest.mark.gpu


def launched(call, path):
    """The names of the library's kernels that the call launches."""
    call()                                               # (one-time set-up)
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as p:
        torch.zeros(1, device="cuda")
        call()
        torch.cuda.synchronize()
    p.export_chrome_trace(path)
    with open(path) as f:
        names = [e["name"] for e in json.load(f)["traceEvents"] if e.get("cat") == "kernel"]
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


PRODUCTS = [
    (20, 2048, 2048, 0, "gemm_i8_skinny_kernel<32, 0>"), (33, 1024, 2048, 1, "gemm_i8_skinny_kernel<64, 1>"), (100, 1024, 2048, 2, "gemm_i8_skinny_kernel<128, 2>"),
    (971, 9728, 896, 1, "gemm_i8_kernel<192, 1>"), (8192, 4096, 2048, 0, "gemm_i8_pair_kernel<0>"), (300, 64, 40, 0, "gemm_i8_simt_kernel<__nv_bfloat16, false>")]
ROWS = [("bf16", 20, 2048, "quantize_rows_kernel<__nv_bfloat16, 128, true>"), ("fp32", 7, 33, "quantize_rows_kernel<float, 32, false>"),
        ("bf16", 16008, 1024, "quantize_stream_kernel<__nv_bfloat16, 32>"), ("fp32", 2000, 11008, "quantize_stream_kernel<float, 512>")]


def attention(dtype, hd, news, form, page):
    from paged_helpers import Paged, engine
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = torch.full((1,), 0.1, device="cuda")
    p = Paged(dtype, news, [n + 20 for n in news], 1, 1, hd, page)
    eng, kv, q = engine(dtype), p.kv(), p.q.cuda()
    return lambda: eng.paged_attention(kv, q, **form)


def product(M, N, K, epilogue):
    from paged_helpers import engine
    eng = engine("bf16")
    a, w = (torch.ones(n, K, dtype=torch.int8, device="cuda") for n in (M, N))
    sa, sw = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    out = torch.zeros(M, N, dtype=torch.float32 if epilogue else torch.bfloat16, device="cuda")
    return lambda: eng.gemm_int8(a, sa, w, sw, out, epilogue=epilogue)


def rows(dtype, M, K):
    from paged_helpers import engine
    eng = engine(dtype)
    x = torch.ones(M, K, dtype=eng.dtype, device="cuda")
    return lambda: eng.quantize_rows(x)


CALLS = [(f, c[:-1], c[-1]) for f, cases in ((attention, ATTENTION), (product, PRODUCTS), (rows, ROWS)) for c in cases]


@pytest.fixture(scope="module")
def names():
    """What each call launches, from a process of its own: after some minutes of a session the profiler drops records."""
    done = subprocess.run([sys.executable, os.path.abspath(__file__)], capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stderr[-3000:]
    return json.loads(done.stdout.splitlines()[-1])


@pytest.mark.parametrize("i", range(len(CALLS)), ids=[c[2] for c in CALLS])
def test_the_kernel_of_a_call(names, i):
    if not any(names):
        pytest.skip("no activity records: another profiler holds the process")
    assert [n for n in names[i] if "join" not in n] == [CALLS[i][2]], names[i]


if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    with tempfile.TemporaryDirectory() as d:
        print(json.dumps([launched(f(*args), os.path.join(d, "trace.json")) for f, args, _ in CALLS]))
