"""Calls without rows, as a step makes them in which no sequence has a new one: served, and nothing is touched."""
import pytest
import torch

from paged_helpers import Paged, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64), ("bf16", 128)])
def test_append_and_attention(dtype, hd):
    from paper_2511_18793_b200 import binding
    eng = engine(dtype)
    p = Paged(dtype, [0, 0], [40, 0], 4, 2, hd, 16, garbage=1.0)
    k_before, v_before = p.k_pool.clone(), p.v_pool.clone()
    x = torch.randn(6, 8, hd, device="cuda").to(p.dt)
    none = x[6:]
    tab = eng.rope_table(binding.Rope(hd), 64)
    for bounds in (dict(), dict(max_new=3), dict(max_new=0)):
        kv = p.kv(**bounds)
        for rope in (None, tab):
            q = eng.kv_append(kv, none[:, 4:6], none[:, 6:], q=none[:, :4], rope=rope)
            assert tuple(q.shape) == (0, 4, hd)
            assert eng.kv_append(kv, none[:, 4:6], none[:, 6:], rope=rope) is None
        for form in (dict(), dict(causal=False), dict(window=5, softcap=3.0)):
            out = eng.paged_attention(kv, q, lse=torch.empty(0, 4, device="cuda"), **form)
            assert tuple(out.shape) == (0, 4, hd)
    eng.sync()
    assert torch.equal(p.k_pool, k_before) and torch.equal(p.v_pool, v_before)


def test_an_empty_rotary_table():
    from paper_2511_18793_b200 import binding
    assert tuple(engine("bf16").rope_table(binding.Rope(64), 0).table.shape) == (0, 64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_to_8_bits_and_products(dtype):
    eng = engine(dtype)
    w, ws = torch.ones(32, 64, dtype=torch.int8, device="cuda"), torch.ones(32, device="cuda")
    q, s = eng.quantize_rows(torch.empty(0, 64, dtype=eng.dtype, device="cuda"))
    assert tuple(q.shape) == (0, 64) and tuple(s.shape) == (0,)
    for epilogue, t in ((0, eng.dtype), (1, torch.float32), (2, torch.float32)):
        out = torch.empty(0, 32, dtype=t, device="cuda")
        assert eng.gemm_int8(q, s, w, ws, out, epilogue=epilogue) is out
    eng.sync()


def test_other_arguments_are_still_looked_at():
    from paper_2511_18793_b200 import binding
    eng = engine("bf16")
    lib, h = binding.lib, eng._h
    assert lib.nezha_quantize_rows(h, None, 64, 0, 64, None, None) == 0
    assert lib.nezha_quantize_rows(h, None, 63, 0, 64, None, None) == 1 and lib.nezha_quantize_rows(h, None, 64, -1, 64, None, None) == 1
    p = Paged("bf16", [0], [40], 4, 2, 64, 16)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    for form in (dict(softcap=-1.0), dict(window=-1)):
        with pytest.raises(binding.NezhaError) as e:
            eng.paged_attention(p.kv(), none, **form)
        assert e.value.status == 1
    with pytest.raises(binding.NezhaError) as e:
        eng.kv_append(p.kv(max_kv=49), none[:, :2], none[:, 2:])
    assert e.value.status == 1
    eng.sync()
