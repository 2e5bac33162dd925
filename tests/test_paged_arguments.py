"""What the binding passes on for a paged cache, on tensors that stand in for a GPU's (no launch is made)."""
import torch

from paper_2511_18793_b200 import binding


class OnGpu(torch.Tensor):
    """A CPU tensor that says it is on GPU 0."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def on_gpu(t):
    return t.as_subclass(OnGpu)


def paged(table=None, batch=3, **kw):
    pool = on_gpu(torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16))
    table = on_gpu(torch.zeros(batch, 4, dtype=torch.int32)) if table is None else table
    start, length = (on_gpu(torch.zeros(n, dtype=torch.int32)) for n in (table.shape[0] + 1, table.shape[0]))
    return binding.PagedKV(pool, pool, table, start, length, **kw)


def described(kv, rows):
    return kv._for(rows)._obj


def test_the_stride_of_a_table_is_its_own():
    wide = on_gpu(torch.zeros(3, 9, dtype=torch.int32))
    assert described(paged(wide), 1).table_stride == 9
    assert described(paged(wide[:, :4]), 1).table_stride == 9 and described(paged(wide[:, :4]), 1).max_pages == 4
    # one history's pages for all sequences: rows of a table that lie on one another
    assert described(paged(wide[:1, :4].expand(3, 4)), 1).table_stride == 0
    # sequences one page apart in a longer list
    assert described(paged(on_gpu(torch.zeros(20, dtype=torch.int32)).as_strided((3, 4), (1, 1))), 1).table_stride == 1
    # of one sequence it does not matter
    assert described(paged(wide[:1, :4].expand(1, 4)), 1).table_stride >= 0


def test_attributes_that_are_set():
    kv = paged()
    assert kv.max_kv == 4 * 16 and kv.max_new is None
    first = described(kv, 5)
    assert (first.max_kv, first.max_new, first.rows) == (64, 5, 5) and described(kv, 5) is first
    kv.max_kv, kv.max_new = 40, 2
    assert (described(kv, 5).max_kv, described(kv, 5).max_new) == (40, 2) and (first.max_kv, first.max_new) == (64, 5)
    kv.max_kv = None
    kv.page_table = on_gpu(torch.zeros(3, 7, dtype=torch.int32))
    assert kv.max_kv == 7 * 16 == described(kv, 5).max_kv and described(kv, 5).max_pages == 7
    kv.kv_len += 1                                   # the same tensor
    assert described(kv, 5).kv_len == kv.kv_len.data_ptr()
    lens = kv.kv_len = on_gpu(torch.ones(3, dtype=torch.int32))
    assert described(kv, 5).kv_len == lens.data_ptr()
