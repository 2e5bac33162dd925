"""Products too large for one call are refused before anything is launched."""
import pytest
import torch

from paged_helpers import engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N", [(2 ** 31 - 1, 1), (1, 2 ** 31 - 1), (2 ** 31 - 255, 1), (1, 2 ** 31 - 255), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 24, 2 ** 24)])
@pytest.mark.parametrize("K", [16, 7])
def test_products(M, N, K):
    from paper_2511_18793_b200 import binding
    eng = engine("bf16")
    a, s, c = torch.zeros(64, dtype=torch.int8, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    st = binding.lib.nezha_gemm_int8(eng._h, a.data_ptr(), s.data_ptr(), a.data_ptr(), s.data_ptr(), c.data_ptr(), M, N, K, 1, None)
    assert st == 7
    eng.sync()
