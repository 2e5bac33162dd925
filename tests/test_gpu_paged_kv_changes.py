"""What a description of a paged cache says is what its attributes say at the time of the call."""
import pytest
import torch

from paged_helpers import Paged, engine, reference

pytestmark = pytest.mark.gpu


def served(eng, p, kv):
    out = eng.paged_attention(kv, p.q.cuda())
    eng.sync()
    want, _, tol = reference(p)
    return bool(((out.double().cpu() - want).abs() <= tol).all())


def shorter(p, lens):
    """The same pool and new rows on the first positions only."""
    s = Paged(p.dtype, p.news, p.lens, p.hq, p.hkv, p.hd, p.page)
    s.lens, s.k, s.v = lens, [k[:n] for k, n in zip(p.k, lens)], [v[:n] for v, n in zip(p.v, lens)]
    s.k_pool, s.v_pool, s.d_table, s.q = p.k_pool, p.v_pool, p.d_table, p.q
    s.kv_len = torch.tensor(lens, dtype=torch.int32).cuda()
    return s


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64)])
def test_bounds_that_grow(dtype, hd):
    from paper_2511_18793_b200 import binding
    eng = engine(dtype)
    p = Paged(dtype, [2, 4], [300, 77], 4, 2, hd, 16)
    s = shorter(p, [40, 30])
    kv = binding.PagedKV(p.k_pool, p.v_pool, p.d_table, p.row_start, s.kv_len, 4, 40)
    assert served(eng, s, kv)
    s.kv_len.copy_(torch.tensor(p.lens, dtype=torch.int32))       # the context grows in place, and the bound with it
    kv.max_kv = 300
    assert served(eng, p, kv)
    kv.max_new = 3                                                # fewer rows than the second sequence has
    with pytest.raises(binding.NezhaError) as e:
        served(eng, p, kv)
    assert e.value.status == 8
    kv.max_new = None
    assert served(eng, p, kv)


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64)])
def test_tensors_that_are_replaced(dtype, hd):
    from paper_2511_18793_b200 import binding
    eng = engine(dtype)
    p = Paged(dtype, [2, 4], [300, 77], 4, 2, hd, 16)
    s = shorter(p, [40, 30])
    kv = binding.PagedKV(p.k_pool, p.v_pool, p.d_table, p.row_start, s.kv_len, 4, 300)
    assert served(eng, s, kv)
    kv.kv_len = p.kv_len                                          # other lengths
    assert served(eng, p, kv)
    other = Paged(dtype, [4, 2], [200, 100], 4, 2, hd, 16, seed=3)
    kv.k_pool = other.k_pool                                      # all of it, one after the other
    kv.v_pool = other.v_pool
    kv.page_table, kv.row_start, kv.kv_len = other.d_table, other.row_start, other.kv_len
    kv.max_kv = 200
    assert served(eng, other, kv)
    kv.kv_len -= 1                                                # in place
    t = shorter(other, [199, 99])
    assert served(eng, t, kv)


def test_what_does_not_fit_is_refused():
    from paper_2511_18793_b200 import binding
    eng = engine("bf16")
    p = Paged("bf16", [2, 4], [30, 77], 4, 2, 64, 16)
    kv, q = p.kv(), p.q.cuda()
    kv.kv_len = p.kv_len[:1]
    with pytest.raises(AssertionError):
        eng.paged_attention(kv, q)
    kv.kv_len = p.kv_len.long()
    with pytest.raises(AssertionError):
        eng.paged_attention(kv, q)
    kv.kv_len = p.kv_len
    kv.v_pool = p.v_pool.float()
    with pytest.raises(AssertionError):
        eng.paged_attention(kv, q)
    kv.v_pool = p.v_pool
    assert served(eng, p, kv)
    kv.max_kv = p.d_table.shape[1] * 16 + 1
    with pytest.raises(binding.NezhaError) as e:
        eng.paged_attention(kv, q)
    assert e.value.status == 1
