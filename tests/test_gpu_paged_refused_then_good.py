"""A refused call leaves nothing behind that a good one on the same description would use."""
import math

import pytest
import torch

from paged_helpers import Paged, engine, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("refused", [dict(softcap=-1.0), dict(scale=math.inf), dict(softcap=2e30), dict(softcap=math.nan)])
def test_a_good_call_behind_a_refused_one(hd, refused):
    """One token of a long context: the good call needs a workspace."""
    from paper_2511_18793_b200 import binding
    p = Paged("bf16", [1], [5003], 8, 2, hd, 16)
    eng, kv, q = engine("bf16"), p.kv(), p.q.cuda()
    for _ in range(2):
        with pytest.raises(binding.NezhaError) as e:
            eng.paged_attention(kv, q, **refused)
        assert e.value.status == 1
    out = eng.paged_attention(kv, q)
    eng.sync()
    want, _, tol = reference(p)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
    assert torch.equal(out, eng.paged_attention(p.kv(), q))
    eng.sync()
