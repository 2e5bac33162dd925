"""Pages that have left every row's window may be given back: their entries of the table are not looked at."""
import pytest
import torch

from paged_helpers import Paged, engine
from test_gpu_paged_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("fp32", 32), ("fp32", 64), ("fp32", 128), ("bf16", 16), ("bf16", 32), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("page", [1, 8, 16, 20])
@pytest.mark.parametrize("new", [1, 5, 30, 140])
def test_pages_in_front_of_the_window(dtype, hd, page, new):
    for length, window in ((new + 200, 50), (new + 77, 41), (new + 1000, 333)):
        p = Paged(dtype, [new], [length], 4, 2, hd, page)
        first_seen = length - new - window + 1
        p.d_table[0, : max(0, first_seen // page)] = -1
        torch.cuda.synchronize()
        check(p, dict(window=window), rows=sorted({0, new // 2, new - 1}))     # (synchronises: a bad page would be reported)
    engine(dtype).sync()
