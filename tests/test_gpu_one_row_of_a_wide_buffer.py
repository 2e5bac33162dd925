"""One row cut out of rows of any length: the distance to the next row, which there is not, is not looked at."""
import pytest
import torch

from paged_helpers import Paged, engine, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64)])
def test_append_and_attention(dtype, hd):
    p = Paged(dtype, [1], [50], 4, 2, hd, 16)
    eng = engine(dtype)
    wide = torch.zeros(3, 8 * hd + 1, dtype=p.dt, device="cuda")
    x = wide[:, : 8 * hd].unflatten(1, (8, hd))[:1]
    assert x.stride(0) % 2 == 1
    x[:, :4] = p.q.cuda()
    x[:, 4:6], x[:, 6:] = p.k[0][-1:].cuda(), p.v[0][-1:].cuda()
    kv = p.kv()
    torch.cuda.synchronize()
    q = eng.kv_append(kv, x[:, 4:6], x[:, 6:], q=x[:, :4])
    out = torch.zeros(2, 4 * hd + 3, dtype=p.dt, device="cuda")[:, : 4 * hd].unflatten(1, (4, hd))[:1]
    torch.cuda.synchronize()
    eng.paged_attention(kv, x[:, :4], out=out)
    eng.sync()
    assert torch.equal(q.cpu(), p.q)
    want, _, tol = reference(p)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
