"""Attention of more rows than one call counts is refused before anything is launched."""
import ctypes as C

import pytest
import torch

from paged_helpers import Paged, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64)])
@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 1023])
def test_rows_next_to_two_to_the_31(dtype, hd, rows):
    from paper_2511_18793_b200 import binding
    p = Paged(dtype, [1], [20], 1, 1, hd, 16)
    eng, kv, q = engine(dtype), p.kv(), p.q.cuda()
    out = torch.full_like(q, 5.0)
    desc = binding.NezhaPagedKV(*kv._fields, rows, rows, 20)
    form = binding.NezhaAttnForm(1, 0, 1.0, 0.0, None)
    st = binding.lib.nezha_paged_attention(eng._h, C.byref(desc), q.data_ptr(), hd, 1, C.byref(form), out.data_ptr(), hd, None, None, 0)
    assert st == 1 and binding.lib.nezha_paged_attention_workspace(eng._h, C.byref(desc), 1, C.byref(form)) == 0
    eng.sync()
    assert bool((out == 5.0).all())
