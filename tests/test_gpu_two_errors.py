"""Errors of two kinds before one synchronising call: a wait that gave up is not hidden by a bad page."""
import pytest
import torch

from paged_helpers import Paged, engine

pytestmark = pytest.mark.gpu


def test_a_wait_that_gave_up_and_a_bad_page():
    from paper_2511_18793_b200 import binding
    eng = engine("bf16")
    p = Paged("bf16", [2], [40], 4, 2, 64, 16)
    p.d_table[0, 1] = -1
    q = p.q.cuda()
    eng.sync()
    torch.cuda.synchronize()
    words = eng.arena[: eng.arena.numel() // 4 * 4].view(torch.int32)
    before = words.clone()
    eng.paged_attention(p.kv(), q)
    torch.cuda.synchronize()
    at = torch.nonzero(words != before).flatten()
    assert at.numel() == 1 and int(before[at]) == 0 and int(words[at]) == 8      # the status word, with the bit of a bad page
    words[at] = 8 | 4                                                             # and that of a wait that gave up
    torch.cuda.synchronize()
    with pytest.raises(binding.NezhaError) as e:
        eng.sync()
    assert e.value.status == 4 and "wait" in str(e.value) and "page" in str(e.value)
    eng.sync()                                                                    # reported once
    eng.paged_attention(p.kv(), q)
    with pytest.raises(binding.NezhaError) as e:
        eng.sync()
    assert e.value.status == 8
    eng.sync()
