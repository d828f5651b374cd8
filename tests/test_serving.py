"""Page plans, draws and cross-attention over pages without a GPU: the oracle's own pins, and what the entry points refuse before anything is enqueued."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import serving as O

EINVAL, ESHAPE, ENULL = -1, -2, -3


@pytest.fixture(scope="module")
def L():
    import paper_2312_11462_amd as P
    if not os.path.exists(P.library_path()):
        from paper_2312_11462_amd import build
        build.build()
    return P.lib()


# ------------------------------------------------------------------------------------------------ the oracle

def test_oracle_weights_are_the_softmax_where_nothing_is_left_out():
    x = np.random.default_rng(1).standard_normal(300) * 3
    w, _ = O.weights(x, 0.7)
    assert np.allclose(w / w.sum(), torch.softmax(torch.tensor(x) / 0.7, -1).numpy(), rtol=1e-13)


def test_oracle_keeps_what_the_parameters_say():
    p = np.array([0.1, 0.4, 0.05, 0.4, 0.05])
    x = np.log(p)
    assert np.flatnonzero(O.weights(x, top_k=1)[0]).tolist() == [1]                      # of equal ones the lowest
    assert np.flatnonzero(O.weights(x, top_k=4)[0]).tolist() == [0, 1, 2, 3]
    assert np.flatnonzero(O.weights(x, top_p=0.45)[0]).tolist() == [1, 3]
    assert np.flatnonzero(O.weights(x, top_p=0.0)[0]).tolist() == [1]
    assert np.flatnonzero(O.weights(x, top_p=0.85)[0]).tolist() == [0, 1, 3]
    assert np.flatnonzero(O.weights(x, min_p=0.2)[0]).tolist() == [0, 1, 3]
    assert np.flatnonzero(O.weights(x, top_k=3, top_p=0.88)[0]).tolist() == [1, 3]       # 0.8 of the three's 0.9
    assert np.flatnonzero(O.weights(x, temperature=0.0)[0]).tolist() == [1]
    assert O.weights(np.full(4, -np.inf))[0].tolist() == [0, 0, 0, 0]
    assert O.weights(np.array([np.nan, np.inf, 3.0, np.inf]))[0].tolist() == [0, 1, 0, 1]


def test_oracle_draws_have_the_law_of_the_weights():
    w = np.array([0.25, 0.0, 0.5, 0.25])
    u = (np.arange(1 << 12) + 0.0) / (1 << 12)
    assert np.bincount([O.draw(w, x) for x in u], minlength=4).tolist() == [1024, 0, 2048, 1024]
    assert O.draw(w, 1.0) == 3 and O.draw(w, 0.0) == 0 and O.draw(np.zeros(3), 0.5) == -1


def test_oracle_pages_go_round():
    p = O.Pages([[-1] * 4 for _ in range(3)], [0, 0, 0], list(range(9, -1, -1)), [0] * 10, 16)
    row_start, seq, pos, slot, served = p.plan([0, 0, 0], [20, 1, 70], 128)
    assert served == [1, 1, 0] and row_start == [0, 20, 21, 21]                          # 70 rows: five pages, the table has four
    assert p.table[0][:2] == [0, 1] and p.table[1][0] == 2 and slot[19] == 16 + 3 and slot[20] == 32 and slot[21] == seq[21] == pos[21] == -1
    p.share([-1, -1, 0], [0, 0, 31])
    assert p.table[2][:1] == [0] and p.held == [2, 1, 1] and p.users[:3] == [2, 1, 1]
    p.release([0, -1, 0])
    assert p.free[-2:] == [1, 0] and p.held == [0, 1, 0] and p.users == [0, 0, 1] + [0] * 7
    assert p.plan([0, 1, 0], [17, 0, 0], 17)[4] == [1, 1, 1] and p.table[0][:2] == [0, 1]


def test_oracle_cross_attention_is_softmax_attention_over_the_states():
    rng = np.random.default_rng(4)
    n, m, kv, g, d, page = 21, 3, 2, 3, 16, 16
    dense_k, dense_v = rng.standard_normal((n, kv, d)), rng.standard_normal((n, kv, d))
    k, v = np.full((5, kv, page, d), np.nan), np.full((5, kv, page, d), np.nan)
    for j in range(n):
        k[[4, 1][j // page], :, j % page], v[[4, 1][j // page], :, j % page] = dense_k[j], dense_v[j]
    q = rng.standard_normal((m, kv * g, d))
    out = O.cross_attention(k, v, np.array([[4, 1]]), [0, m], [n], q, 0.25)
    t = [torch.tensor(x).transpose(0, 1)[None] for x in (q, dense_k.repeat(g, 1), dense_v.repeat(g, 1))]
    assert np.allclose(out, torch.nn.functional.scaled_dot_product_attention(*t, scale=0.25)[0].transpose(0, 1).numpy(), rtol=1e-12, atol=1e-13)


# ------------------------------------------------------------------------------------------------ refusals

def _pages(**change):
    from paper_2312_11462_amd.binding import PageTable
    p = PageTable(8, 16, 2, 4, 256, 256, 256, 256, 256)
    for name, value in change.items():
        setattr(p, name, value)
    return C.addressof(p), p


@pytest.mark.parametrize("change,code", [(dict(table=None), ENULL), (dict(held=None), ENULL), (dict(free_pages=None), ENULL), (dict(n_free=None), ENULL),
                                         (dict(users=None), ENULL), (dict(n_pages=0), EINVAL), (dict(n_sequences=0), EINVAL), (dict(table_stride=0), EINVAL),
                                         (dict(page_rows=8), EINVAL), (dict(page_rows=24), EINVAL), (dict(page_rows=2048), EINVAL),
                                         (dict(table_stride=1 << 27), ESHAPE), (dict(n_sequences=(1 << 20) + 1), ESHAPE),
                                         (dict(n_sequences=1 << 18, table_stride=1 << 13), ESHAPE), (dict(n_pages=(1 << 30) + 1), ESHAPE)], ids=str)
def test_every_page_call_refuses_bad_arrays(L, change, code):
    ref, keep = _pages(**change)
    assert L.csd_pages_plan(ref, 256, 256, 4, 256, 256, 256, 256, 256, None) == code
    assert L.csd_pages_release(ref, 256, None) == code
    assert L.csd_pages_share(ref, 256, 256, None) == code
    assert L.csd_pages_release(None, 256, None) == ENULL


def test_page_calls_refuse_bad_arguments(L):
    ref, keep = _pages()
    good = [256, 256, 4, 256, 256, 256, 256, 256]
    for at, value, code in [(0, None, ENULL), (1, None, ENULL), (2, -1, EINVAL), (2, (1 << 22) + 1, ESHAPE), (3, None, ENULL), (4, None, ENULL),
                            (5, None, ENULL), (6, None, ENULL), (6, 260, EINVAL), (7, None, ENULL)]:
        args = list(good)
        args[at] = value
        assert L.csd_pages_plan(ref, *args, None) == code, (at, value)
    assert L.csd_pages_release(ref, None, None) == ENULL
    assert L.csd_pages_share(ref, None, 256, None) == ENULL
    assert L.csd_pages_share(ref, 256, None, None) == ENULL


def test_draws_refuse_what_they_cannot_do(L):
    from paper_2312_11462_amd.binding import Filter
    nan = float("nan")
    for change, code in [(dict(temperature_all=-1.0), EINVAL), (dict(temperature_all=nan), EINVAL), (dict(top_p_all=-0.5), EINVAL), (dict(top_p_all=nan), EINVAL),
                         (dict(min_p_all=-0.1), EINVAL), (dict(min_p_all=1.5), EINVAL), (dict(min_p_all=nan), EINVAL), (dict(rows_each=0), EINVAL)]:
        f = Filter(None, None, None, None, 1.0, 0, 1.0, 0.0, 1)
        for name, value in change.items():
            setattr(f, name, value)
        assert L.csd_sample(C.addressof(f), 256, 100, 0, 2, 100, 256, 256, None, None) == code, change
        assert L.csd_filter_probs(C.addressof(f), 256, 100, 0, 2, 100, 256, None) == code, change
    f = Filter(None, None, None, None, 1.0, 0, 1.0, 0.0, 1)
    ref = C.addressof(f)
    good = dict(f=ref, x=256, stride=100, dtype=1, rows=2, V=100, probs=1024)
    for change, code in [(dict(f=None), ENULL), (dict(x=None), ENULL), (dict(x=257), EINVAL), (dict(x=258, dtype=0), EINVAL), (dict(stride=99), EINVAL),
                         (dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(V=0), EINVAL), (dict(V=(1 << 18) + 1, stride=1 << 19), ESHAPE),
                         (dict(rows=(1 << 21) + 1), ESHAPE), (dict(probs=1026), EINVAL),
                         (dict(probs=256), EINVAL), (dict(probs=652), EINVAL), (dict(x=1824 - 4), EINVAL)]:
        a = dict(good, **change)
        assert L.csd_filter_probs(a["f"], a["x"], a["stride"], a["dtype"], a["rows"], a["V"], a["probs"], None) == code, change
        assert L.csd_sample(a["f"], a["x"], a["stride"], a["dtype"], a["rows"], a["V"], 256, 256, a["probs"], None) == code, change
    assert L.csd_sample(ref, 256, 100, 1, 2, 100, 1026, 256, None, None) == EINVAL
    assert L.csd_sample(ref, 256, 100, 1, 2, 100, 1024, 258, None, None) == EINVAL
    assert L.csd_sample(ref, 256, 100, 1, 2, 100, None, 256, None, None) == ENULL
    assert L.csd_sample(ref, 256, 100, 1, 2, 100, 256, None, None, None) == ENULL
    assert L.csd_filter_probs(ref, 256, 100, 1, 2, 100, None, None) == ENULL
    # no rows: nothing to do, and no buffers needed
    assert L.csd_sample(ref, None, 100, 1, 0, 100, None, None, None, None) == 0
    assert L.csd_filter_probs(ref, None, 100, 1, 0, 100, None, None) == 0


def test_cross_attention_refuses_what_attention_refuses(L):
    from paper_2312_11462_amd.binding import PagedPool
    pool = PagedPool(2, 8, 16, 4, 64, 2, 256, 256, 256, 256, 256, 4)
    good = dict(p=C.addressof(pool), layer=0, start=256, length=256, B=1, rows=4, max_rows=4, q=256, qs=512, heads=8, dtype=1, scale=0.125, out=256, ws=256)
    for change, code in [(dict(p=None), ENULL), (dict(layer=2), EINVAL), (dict(start=None), ENULL), (dict(length=None), ENULL), (dict(B=0), EINVAL),
                         (dict(rows=-1), EINVAL), (dict(max_rows=0), EINVAL), (dict(heads=6), EINVAL), (dict(dtype=2), EINVAL), (dict(q=None), ENULL),
                         (dict(out=None), ENULL), (dict(ws=None), ENULL), (dict(qs=504), EINVAL), (dict(q=264), EINVAL), (dict(out=264), EINVAL),
                         (dict(ws=128), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(heads=4 << 20, qs=1 << 28), ESHAPE)]:
        a = dict(good, **change)
        assert L.csd_paged_cross_attention(a["p"], a["layer"], a["start"], a["length"], a["B"], a["rows"], a["max_rows"], a["q"], a["qs"], a["heads"],
                                           a["dtype"], a["scale"], a["out"], a["ws"], None) == code, change
    assert L.csd_paged_cross_attention(good["p"], 0, 256, 256, 1, 0, 1, None, 0, 8, 1, 0.125, None, None, None) == 0


def test_the_binding_refuses_tensors_of_the_host():
    import paper_2312_11462_amd as P
    with pytest.raises(ValueError):
        P.sample(torch.zeros(2, 8), torch.zeros(2))
    with pytest.raises(ValueError):
        P.filter_probs(torch.zeros(2, 8))
    with pytest.raises(ValueError):
        P.Pages.new(4, 16, 2, 2, device="cpu")


def test_rows_of_any_leading_dimensions():
    from paper_2312_11462_amd.binding import _rows_of
    for shape in ((7,), (3, 7), (2, 3, 7), (2, 1, 3, 7), (1, 1, 7)):
        x = torch.zeros(shape)
        rows = x.numel() // 7
        assert _rows_of(x.shape, x.stride()) == (rows, 7)
    for shape in ((0, 7), (2, 0, 7), (0, 2, 7), (2, 0, 3, 7)):
        assert _rows_of(shape, torch.zeros(shape).stride())[0] == 0
    wide = torch.zeros(2, 3, 11)[..., :7]
    assert _rows_of(wide.shape, wide.stride()) == (6, 11)
    for x in (torch.zeros(2, 4, 7)[:, :3], torch.zeros(3, 7, 2)[..., 0], torch.zeros(()), torch.zeros(3, 0)):
        with pytest.raises(ValueError):
            _rows_of(x.shape, x.stride())


def test_oracle_rows_of_shared_pages_are_nobodys_to_write():
    p = O.Pages([[-1] * 5 for _ in range(3)], [0, 0, 0], list(range(11, -1, -1)), [0] * 12, 16)
    p.plan([0, 0, 0], [48, 0, 0], 48)
    p.share([-1, 0, -1], [0, 48, 0])
    p.release([-1, 40, -1])                                  # the one that took the pages is cut inside the last of them
    assert p.users[:3] == [2, 2, 2]
    before = [list(r) for r in p.table], list(p.held), list(p.free), list(p.users)
    row_start, seq, pos, slot, served = p.plan([48, 40, 0], [1, 8, 2], 16)
    assert served == [1, 0, 1] and row_start == [0, 1, 1, 3] and slot[:4] == [48, 64, 65, -1]      # it counts for nothing, and keeps what it holds
    assert p.table[1] == before[0][1] and p.held[1] == 3 and p.users[:5] == [2, 2, 2, 1, 1]
    assert p.plan([48, 40, 0], [0, 0, 0], 4)[4] == [1, 1, 1]                                       # without rows there is nothing to write
    p.release([40, -1, 0])                                   # and the one that gave them
    assert p.plan([40, 40, 0], [3, 3, 3], 16)[4] == [0, 0, 1]
    p.release([-1, 32, 0])                                   # back to the page's first row: the rows from there on go to a page of its own
    row_start, seq, pos, slot, served = p.plan([40, 32, 0], [3, 16, 0], 19)
    assert served == [1, 1, 1] and slot[:3] == [40, 41, 42] and p.users[:3] == [2, 2, 1] and p.table[1][2] == slot[3] // 16 not in p.table[0][:3]
    assert p.plan([10, 8, 0], [30, 100, 0], 130)[4] == [0, 0, 1]                                   # (100 rows do not fit its table; the 30 begin in a shared page)
    p.release([-1, 0, -1])
    assert p.plan([10, 0, 0], [30, 0, 0], 30)[4] == [1, 1, 1]


def test_draws_refuse_rows_that_their_parameters_do_not_cover(L):
    """Five rows by two: the arrays have two entries, and the last row would read a third."""
    from paper_2312_11462_amd.binding import Filter
    for name in ("temperature", "top_k", "top_p", "min_p"):
        for rows, each in ((5, 2), (1, 2), (7, 3), (2, 1 << 30)):
            f = Filter(None, None, None, None, 1.0, 0, 1.0, 0.0, each)
            setattr(f, name, 256)
            assert L.csd_sample(C.addressof(f), 256, 100, 1, rows, 100, 256, 256, None, None) == EINVAL, (name, rows, each)
            assert L.csd_filter_probs(C.addressof(f), 256, 100, 1, rows, 100, 4096, None) == EINVAL, (name, rows, each)
            assert L.csd_sample(C.addressof(f), None, 100, 1, 0, 100, None, None, None, None) == 0


def test_numbers_that_the_parameters_types_do_not_hold():
    """A top_k beyond int32 is more than there are; numbers beyond fp32 are its largest; what is no number is said to be none."""
    import math
    from paper_2312_11462_amd.binding import _in_range
    big = float(np.finfo(np.float32).max)
    assert _in_range([1e39, 2 ** 40, 1e300, 0.0]) == [big, 2 ** 31 - 1, big, 0.0]
    assert _in_range([math.inf, -2 ** 70, 1, -1e39]) == [math.inf, 0, 1.0, -big]
    assert math.isnan(_in_range([math.nan, 2 ** 40, 1.0, 0.0])[0])
    for at, bad in ((0, "warm"), (1, 5.5), (1, None), (2, [0.5]), (3, 10 ** 400)):
        numbers = [1.0, 0, 1.0, 0.0]
        numbers[at] = bad
        with pytest.raises(TypeError):
            _in_range(numbers)
