"""The operators take tensors of the engine's GPU only: a launch goes there, whatever GPU a tensor is on.  (Stand-ins for GPU tensors; no launch is made.)"""
import pytest
import torch

from paper_2511_18793_b200 import binding
from test_paged_arguments import OnGpu, on_gpu


class OnOther(OnGpu):
    """The same on GPU 1."""

    def get_device(self):
        return 1


class Lib:
    """Every call is well."""

    def __getattr__(self, name):
        return lambda *a: 0


@pytest.fixture
def eng(monkeypatch):
    monkeypatch.setattr(binding, "lib", Lib())
    e = object.__new__(binding.Engine)
    e._dev, e._dtype, e._h = 0, torch.bfloat16, None
    return e


def rows(heads):
    return on_gpu(torch.zeros(5, heads, 64, dtype=torch.bfloat16))


def whole(*shape):
    return on_gpu(torch.zeros(*shape, dtype=torch.int32))


def floats(*shape):
    return on_gpu(torch.zeros(*shape))


def bytes8(*shape):
    return on_gpu(torch.zeros(*shape, dtype=torch.int8))


def append(e, t):
    kv = binding.PagedKV(t["pool"], t["pool"], t["page_table"], t["row_start"], t["kv_len"])
    return e.kv_append(kv, t["k"], t["v"], q=t["q"], q_out=t["q_out"], rope=binding.RopeTable(binding.Rope(64), t["table"]), positions=t["positions"])


def attend(e, t):
    kv = binding.PagedKV(t["pool"], t["pool"], t["page_table"], t["row_start"], t["kv_len"])
    return e.paged_attention(kv, t["q"], slopes=t["slopes"], out=t["out"], lse=t["lse"])


def cache():
    return dict(pool=on_gpu(torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16)), page_table=whole(3, 4), row_start=whole(4), kv_len=whole(3))


CALLS = {
    "append": (append, lambda: dict(cache(), q=rows(4), k=rows(2), v=rows(2), q_out=rows(4), table=floats(9, 64), positions=whole(5)), ("page_table", "row_start", "kv_len")),
    "attend": (attend, lambda: dict(cache(), q=rows(4), out=rows(4), slopes=floats(4), lse=floats(5, 4)), ("page_table", "row_start", "kv_len")),
    "quantize": (lambda e, t: e.quantize_rows(t["x"], q=t["q"], scale=t["scale"]),
                 lambda: dict(x=on_gpu(torch.zeros(5, 64, dtype=torch.bfloat16)), q=bytes8(5, 64), scale=floats(5)), ()),
    "product": (lambda e, t: e.gemm_int8(t["A"], t["a_scale"], t["W"], t["w_scale"], t["C"], epilogue=1, bias=t["bias"]),
                lambda: dict(A=bytes8(5, 64), a_scale=floats(5), W=bytes8(7, 64), w_scale=floats(7), C=floats(5, 7), bias=floats(7)), ()),
}


@pytest.mark.parametrize("call", sorted(CALLS))
def test_a_tensor_of_another_gpu_is_refused(eng, call):
    run, tensors, with_pool = CALLS[call]
    run(eng, tensors())
    for name in tensors():
        if name in with_pool:
            continue                                 # (compared with the pool's device by the description itself)
        t = tensors()
        t[name] = t[name].as_subclass(OnOther)
        with pytest.raises(AssertionError):
            run(eng, t)
    t = {k: v.as_subclass(OnOther) for k, v in tensors().items()}
    with pytest.raises(AssertionError):
        run(eng, t)
