"""Attention over a paged cache at the borders of its kernels: numbers of rows, interior tiles between edges, forms over many rows."""
import pytest
import torch

from paged_helpers import Paged
from test_gpu_paged_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [1, 8, 9, 16, 17, 64, 65, 128, 129, 256, 257, 384, 385, 512, 513])
def test_numbers_of_rows(hd, rows):
    """One query head per KV head, so a new token is a row; a context that ends inside a tile."""
    p = Paged("bf16", [rows], [rows + 77], 1, 1, hd, 16, tail_rows=1)
    some = sorted({0, rows // 2, max(0, rows - 130), rows - 1} | set(range(max(0, rows - 3), rows)) | {min(rows - 1, t) for t in (63, 64, 127, 128, 255, 256)})
    check(p, rows=some)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("length", [1, 63, 64, 65, 128, 129, 192, 256, 257, 385])
@pytest.mark.parametrize("new", [20, 150])
def test_numbers_of_tiles(hd, length, new):
    """All rows see all of a context of one, two, three and more tiles, which is shorter than the rows too."""
    p = Paged("bf16", [min(new, length)], [length], 6, 1, hd, 16)
    n = min(new, length)
    check(p, dict(causal=False), rows=sorted({0, n // 2, n - 1}))


# (query heads, KV heads, new tokens): 124 and 128 rows, 256, 280, 516 (four of them in a tile of their own)
MANY = [(4, 1, 31), (8, 2, 32), (4, 1, 64), (4, 1, 70), (8, 2, 129)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("hq,hkv,new", MANY)
@pytest.mark.parametrize("form", [dict(window=1000), dict(window=1500, softcap=30.0), dict(window=700, slopes=True), dict(window=1111, softcap=50.0, slopes=True), dict()])
def test_interior_tiles_between_edges(hd, hq, hkv, new, form):
    """What lies outside the windows is NaN, and so is what the tiles on the edges hold that nobody sees."""
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = torch.tensor([2.0 ** -(1 + h) for h in range(hq)])
    lens = [2900, new + 1]
    p = Paged("bf16", [new, min(new, 40)], lens, hq, hkv, hd, 32)
    window = form.get("window", 0)
    if window:                                           # pages that no row of the first sequence sees
        first_seen = lens[0] - new - window + 1
        for page in range(first_seen // 32):
            p.k_pool[int(p.table[0, page])] = float("nan")
            p.v_pool[int(p.table[0, page])] = float("inf")
        torch.cuda.synchronize()
    check(p, form, rows=sorted({0, 1, new // 2, new - 2, new - 1, new, new + min(new, 40) - 1}))


@pytest.mark.parametrize("form", [dict(), dict(causal=False), dict(window=500), dict(window=700, softcap=30.0), dict(softcap=4.0, slopes=True),
                                  dict(window=333, slopes=True), dict(window=600, softcap=60.0, slopes=True)])
@pytest.mark.parametrize("hd", [64, 128])
def test_more_tiles_of_rows_than_multiprocessors(hd, form):
    """Up to 516 rows of 64 pairs of a sequence and a KV head, ragged; what nobody sees is NaN."""
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = torch.tensor([2.0 ** -(1 + h) for h in range(8)])
    news = [129, 65, 64, 33, 0, 1] + [129, 100] * 13
    lens = [1400, 1001, 700, 40, 90, 600] + [140, 100] * 13
    p = Paged("bf16", news, lens, 8, 2, hd, 16, tail_rows=1)
    window = form.get("window", 0)
    if window:
        for page in range((lens[0] - news[0] - window + 1) // 16):
            p.k_pool[int(p.table[0, page])] = float("nan")
            p.v_pool[int(p.table[0, page])] = float("inf")
        torch.cuda.synchronize()
    check(p, form, rows=sorted({0, 31, 32, 64, 96, 127, 128, 129, 193, 194, 200, 257, 290, 291, 292, 420, p.starts[-1] - 1}))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new", [1, 4, 14, 30, 60, 130])
@pytest.mark.parametrize("form", [dict(softcap=200.0), dict(softcap=20.0), dict(softcap=1.5), dict(softcap=5.0, scale=-0.2), dict(scale=-0.125),
                                  dict(causal=False, slopes=(0.3, -0.1, 0.0, 0.02)), dict(causal=False, softcap=9.0, slopes=(1.0, 0.004, -0.02, 0.0)),
                                  dict(slopes=(-0.05, 2.0, 30.0, 0.0))])
def test_forms_over_many_rows(hd, new, form):
    """From few rows to many: caps far above the scores, near them and far below; a scale below zero; biases that favour the near, the far and none."""
    form = dict(form)
    if "slopes" in form:
        form["slopes"] = torch.tensor(form["slopes"])
    p = Paged("bf16", [new], [new + 300], 4, 1, hd, 16)
    check(p, form, rows=sorted({0, new // 3, new - 1}))


def test_padded_batches_and_parts():
    """Sequences without rows and without positions among long ones, whose context is dealt out over the GPU."""
    for news, lens in (([1, 0, 1, 0], [5000, 900, 1, 0]), ([0, 0, 2], [0, 7, 9000]), ([30, 0, 1], [6000, 0, 40])):
        check(Paged("bf16", news, lens, 8, 2, 64, 64, tail_rows=2), rows=None if sum(news) < 5 else [0, 15, 29, 30])
        check(Paged("bf16", news, lens, 8, 2, 128, 16, tail_rows=2), dict(causal=False), rows=None if sum(news) < 5 else [0, 15, 29, 30])


@pytest.mark.parametrize("new", [1, 40, 140])
def test_pools_with_room_between(new):
    """Pages inside wider rows of a larger buffer: every stride but the last is free."""
    p = Paged("bf16", [new], [new + 100], 4, 2, 64, 16)
    room = torch.full((p.k_pool.shape[0] + 2, 5, 16, 80), float("nan"), dtype=torch.bfloat16, device="cuda")
    room_v = torch.full_like(room, float("nan"))
    k, v = room[1:-1, 2:4, :, 8:72], room_v[1:-1, 2:4, :, 8:72]
    k.copy_(p.k_pool)
    v.copy_(p.v_pool)
    p.k_pool, p.v_pool = k, v
    torch.cuda.synchronize()
    check(p, rows=sorted({0, new // 2, new - 1}))


def test_positions_end_below_two_to_the_31():
    """A table that repeats one large page describes that many positions; a call that names them all is refused, one of few is served."""
    from paged_helpers import engine
    from paper_2511_18793_b200 import binding
    eng = engine("fp32")
    pool = torch.zeros(1, 1, 2 ** 20, 16, device="cuda")
    table = torch.zeros(1, 2048, dtype=torch.int32, device="cuda")
    start, length = torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda()
    q = torch.ones(1, 1, 16, device="cuda")
    torch.cuda.synchronize()
    with pytest.raises(binding.NezhaError) as e:
        eng.paged_attention(binding.PagedKV(pool, pool, table, start, length, 1, 2 ** 31 - 4095), q)
    assert e.value.status == 1
    out = eng.paged_attention(binding.PagedKV(pool, pool, table, start, length, 1, 2 ** 20), q)
    eng.sync()
    assert bool((out == 0).all())


def test_caps_out_of_range_are_refused_and_those_at_its_ends_served():
    from test_gpu_paged_attention import bad_call
    p = Paged("bf16", [40], [70], 4, 1, 64, 16)
    for kw in (dict(softcap=1e-30), dict(softcap=1e-8, scale=0.125), dict(softcap=2e30), dict(softcap=1.0, scale=2e12), dict(softcap=1e-7, scale=-0.125)):
        bad_call(p, 1, **kw)
    p.q[::2] = 0                                         # rows whose scores are all zero
    check(p, dict(softcap=1.25e-7, scale=0.125))
    check(p, dict(softcap=1e30, scale=0.125))


def test_threads_share_a_description():
    """Calls of different numbers of rows and forms through one PagedKV, from two threads with an engine each."""
    import threading
    from paged_helpers import engine, reference
    p = Paged("bf16", [9], [200], 4, 2, 64, 16)
    few = Paged("bf16", [9], [200], 4, 2, 64, 16)
    few.q = few.q[:, [1, 0, 3, 2]].contiguous()
    few.row_start, few.kv_len, few.d_table, few.k_pool, few.v_pool = p.row_start, p.kv_len, p.d_table, p.k_pool, p.v_pool
    kv = p.kv()
    wants = [reference(p), reference(few, window=30)]
    results, errors = [[], []], []
    engines = [engine("bf16", stream=torch.cuda.Stream()) for _ in range(2)]

    def work(i, q, form):
        try:
            eng = engines[i]
            for n in range(40):
                rows = q if n % 2 else torch.cat([q, q])          # (rows behind the last sequence are left alone)
                results[i].append(eng.paged_attention(kv, rows, **form)[:9])
            eng.sync()
        except Exception as e:                                    # noqa: BLE001
            errors.append(e)

    qs = [p.q.cuda(), few.q.cuda()]
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i, qs[i], f)) for i, f in enumerate((dict(), dict(window=30)))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    torch.cuda.synchronize()
    for got, (want, _, tol) in zip(results, wants):
        for out in got:
            assert bool(((out.double().cpu() - want).abs() <= tol).all())


def test_a_table_of_more_positions_than_an_integer_counts():
    from paged_helpers import engine
    from paper_2511_18793_b200 import binding
    eng = engine("fp32")
    pool = torch.zeros(1, 1, 2 ** 20, 16, device="cuda")
    table = torch.zeros(1, 4096, dtype=torch.int32, device="cuda")
    start, length = torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda()
    torch.cuda.synchronize()
    kv = binding.PagedKV(pool, pool, table, start, length, 1)
    assert kv.max_kv == 2 ** 31 - 4096
    out = eng.paged_attention(kv, torch.ones(1, 1, 16, device="cuda"))
    eng.sync()
    assert bool((out == 0).all())


@pytest.mark.parametrize("dtype,hd", [("fp32", 16), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("new", [6, 40, 150])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 160, 159])
def test_windows_longer_than_every_sequence(dtype, hd, new, window):
    """Next to them: rows in front of their sequence's first position, which see nothing."""
    p = Paged(dtype, [new, new], [new - 5, 160], 2, 1, hd, 16)
    check(p, dict(window=window), rows=sorted({0, 4, 5, 6 % new, new - 1, new, 2 * new - 1}))
