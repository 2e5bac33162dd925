"""As many rows as a call can name."""
import pytest
import torch

from paged_helpers import engine
from test_gpu_int8 import quantized

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("dtype,K", [("bf16", 8), ("fp32", 4), ("bf16", 1), ("fp32", 1)])
def test_rows_to_8_bits(dtype, K):
    """The ring of rows in shared memory (K = 8, 4) and a warp per row."""
    eng = engine(dtype)
    torch.cuda.empty_cache()
    need = MOST * (K * (eng.dtype.itemsize + 1) + 4)
    if torch.cuda.mem_get_info()[0] < need + 2 ** 32:
        pytest.skip("memory")
    x = torch.zeros(MOST, K, dtype=eng.dtype, device="cuda")
    some = torch.randn(6000, K, generator=torch.Generator().manual_seed(K)).to(eng.dtype)
    for at in (0, 2 ** 30 - 3000, MOST - 6000):
        x[at: at + 6000] = some.cuda()
    q, s = torch.full((MOST, K), 99, dtype=torch.int8, device="cuda"), torch.full((MOST,), 7.0, device="cuda")
    torch.cuda.synchronize()
    eng.quantize_rows(x, q=q, scale=s)
    eng.sync()
    want_q, _ = quantized(some)
    want_s = some.float().abs().max(dim=1).values / 127.0
    for at in (0, 2 ** 30 - 3000, MOST - 6000):
        assert torch.equal(q[at: at + 6000].cpu(), want_q) and torch.equal(s[at: at + 6000].cpu(), want_s)
    for lo, hi in ((6000, 2 ** 30 - 3000), (2 ** 30 + 3000, MOST - 6000)):       # rows of zeros
        for i in range(lo, hi, 2 ** 28):
            assert not bool(q[i: min(hi, i + 2 ** 28)].any()) and not bool(s[i: min(hi, i + 2 ** 28)].any())
    del x, q, s
    torch.cuda.empty_cache()
