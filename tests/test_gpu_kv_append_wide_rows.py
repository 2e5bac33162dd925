"""The append of rows of many heads: a row is more than one pass of a block's threads."""
import pytest

from paged_helpers import Paged
from test_gpu_kv_append import check

pytestmark = pytest.mark.gpu

NEWS, LENS = [2, 0, 1, 5], [3, 4, 40, 21]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv", [(64, 64), (96, 96), (128, 128), (129, 43)])
@pytest.mark.parametrize("rope", [None, (64, False), (128, False), (64, True), (128, True)])
def test_rows_of_many_heads(dtype, hq, hkv, rope):
    from paper_2511_18793_b200 import binding
    check(Paged(dtype, NEWS, LENS, hq, hkv, 128, 16, garbage=1.5, tail_rows=1), None if rope is None else binding.Rope(rope[0], interleaved=rope[1]))
