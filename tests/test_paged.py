"""The paged KV cache without a GPU: the oracle's own pins, and what the entry points refuse before anything is enqueued."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

from oracle import paged as O


@pytest.fixture(scope="module")
def L():
    import paper_2312_11462_amd as P
    if not os.path.exists(P.library_path()):
        from paper_2312_11462_amd import build
        build.build()
    return P.lib()


def test_e4m3_rounding_of_the_oracle_is_that_of_the_type():
    g = torch.Generator().manual_seed(5)
    x = torch.cat([(torch.rand(20000, generator=g) - 0.5) * 896, torch.randn(20000, generator=g) * 0.01, torch.tensor([0.0, -0.0, 448.0, -448.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9]),
                   torch.arange(0, 449, 0.5)])
    assert np.array_equal(O.e4m3_round(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())


def test_scale_is_the_smallest_power_that_holds_the_row():
    edges = [448.0, math.nextafter(448.0, 1e9), 224.0, 1.75, 1.7500001, 1.0, 2.0, 3.4e38, 1e-30, 1.2e-38, 1e-45, 0.0]
    for a in edges:
        s = int(O.scale_byte(np.array([[a, -a / 3]]))[0])
        e = s - 127
        assert e >= -126 and a <= 448 * 2.0 ** e and (e == -126 or a > 448 * 2.0 ** (e - 1)), a
    assert int(O.scale_byte(np.array([[np.inf, np.nan, 448.0]]))[0]) == 127


def test_quantised_rows_keep_their_values_when_quantised_again_and_are_near():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((500, 64)) * 10.0 ** rng.uniform(-6, 6, (500, 1))
    y, s = O.quantise(x)
    step = np.exp2(s - 127.0)[:, None]
    assert (np.abs(y - x) <= np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10)).all()
    assert np.array_equal(O.quantise(y)[0], y)


def test_oracle_attention_is_softmax_attention_on_dense_rows():
    rng = np.random.default_rng(4)
    t, m, kv, g, d, page = 21, 6, 2, 3, 16, 16
    dense_k, dense_v = rng.standard_normal((t + m, kv, d)), rng.standard_normal((t + m, kv, d))
    table = np.array([[4, 1]])
    k, v = np.full((5, kv, page, d), np.nan), np.full((5, kv, page, d), np.nan)
    where = O.places([0, t + m], [0], table, page, 5, t + m)
    O.write(k, dense_k, where)
    O.write(v, dense_v, where)
    assert np.array_equal(O.read(k, where, t + m), dense_k)
    q = rng.standard_normal((m, kv * g, d))
    out = O.attention(k, v, table, [0, m], [t], q, 0.25)
    x = torch.einsum("ihd,jhd->hij", torch.tensor(q), torch.tensor(dense_k).repeat_interleave(g, 1)) * 0.25
    x = x.masked_fill(~torch.tril(torch.ones(m, t + m, dtype=torch.bool), t), -math.inf).softmax(-1)
    want = torch.einsum("hij,jhd->ihd", x, torch.tensor(dense_v).repeat_interleave(g, 1)).numpy()
    assert np.allclose(out, want, rtol=1e-12, atol=1e-13)
    # a chain as a tree is the plain block
    assert np.allclose(O.attention(k, v, table, [0, m], [t], q, 0.25, parent=np.arange(m) - 1), want, rtol=1e-12, atol=1e-13)


def _pool(**change):
    from paper_2312_11462_amd.binding import PagedPool
    p = PagedPool(2, 8, 16, 4, 64, 2, 256, 256, 256, 256, 256, 4)
    for name, value in change.items():
        setattr(p, name, value)
    return C.addressof(p), p


EINVAL, ESHAPE, ENULL = -1, -2, -3
POOL_REFUSALS = [(dict(k=None), ENULL), (dict(v=None), ENULL), (dict(table=None), ENULL), (dict(k_scale=None), ENULL), (dict(v_scale=None), ENULL),
                 (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(n_layers=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(n_kv_heads=0), EINVAL),
                 (dict(head_dim=0), EINVAL), (dict(head_dim=12), EINVAL), (dict(head_dim=264), EINVAL), (dict(page_rows=8), EINVAL),
                 (dict(page_rows=24), EINVAL), (dict(page_rows=2048), EINVAL), (dict(table_stride=0), EINVAL), (dict(k=260), EINVAL), (dict(k_scale=257), EINVAL), (dict(v_scale=260), EINVAL),
                 (dict(table_stride=1 << 27), ESHAPE)]


@pytest.mark.parametrize("change,code", POOL_REFUSALS, ids=[str(c[0]) for c in POOL_REFUSALS])
def test_every_call_refuses_a_bad_pool(L, change, code):
    ref, keep = _pool(**change)
    assert L.csd_paged_write(ref, 0, 256, 256, 1, 1, 256, 256, 256, 256, 1, None) == code
    assert L.csd_paged_read(ref, 0, 256, 256, 1, 1, 256, 256, 256, 256, 1, None) == code
    assert L.csd_paged_attention(ref, 0, 256, 256, None, 1, 1, 1, 256, 256, 4, 1, 0.125, 256, 256, None) == code
    assert L.csd_paged_commit(ref, 256, 256, 256, 1, 8, None) == code
    assert L.csd_paged_write(None, 0, 256, 256, 1, 1, 256, 256, 256, 256, 1, None) == ENULL


def test_rows_in_and_out_refuse_what_they_cannot_do(L):
    ref, keep = _pool()
    good = dict(layer=0, start=256, pos=256, B=1, rows=4, k=256, ks=256, v=256, vs=256, dtype=1)
    for change, code in [(dict(layer=2), EINVAL), (dict(layer=-1), EINVAL), (dict(start=None), ENULL), (dict(pos=None), ENULL), (dict(B=0), EINVAL),
                         (dict(rows=-1), EINVAL), (dict(rows=1 << 25), ESHAPE), (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(ks=255), EINVAL),
                         (dict(ks=260), EINVAL), (dict(vs=248), EINVAL), (dict(k=264), EINVAL), (dict(v=258), EINVAL), (dict(dtype=2), EINVAL),
                         (dict(dtype=3), EINVAL), (dict(ks=0), EINVAL), (dict(vs=-256), EINVAL)]:
        a = dict(good, **change)
        args = (ref, a["layer"], a["start"], a["pos"], a["B"], a["rows"], a["k"], a["ks"], a["v"], a["vs"], a["dtype"], None)
        assert L.csd_paged_write(*args) == code, change
        assert L.csd_paged_read(*args) == code, change
    # no rows: nothing to do, and no buffers needed
    assert L.csd_paged_write(ref, 0, 256, 256, 1, 0, None, 0, None, 0, 1, None) == 0
    assert L.csd_paged_read(ref, 0, 256, 256, 1, 0, None, 0, None, 0, 1, None) == 0


def test_attention_refuses_what_it_cannot_do(L):
    ref, keep = _pool()
    good = dict(layer=0, start=256, pos=256, parent=None, B=1, rows=4, max_rows=4, q=256, qs=512, heads=8, dtype=1, scale=0.125, out=256, ws=256)
    for change, code in [(dict(layer=2), EINVAL), (dict(start=None), ENULL), (dict(pos=None), ENULL), (dict(B=0), EINVAL), (dict(rows=-1), EINVAL),
                         (dict(max_rows=0), EINVAL), (dict(heads=6), EINVAL), (dict(heads=0), EINVAL), (dict(dtype=2), EINVAL), (dict(q=None), ENULL),
                         (dict(out=None), ENULL), (dict(ws=None), ENULL), (dict(qs=504), EINVAL), (dict(qs=516), EINVAL), (dict(q=264), EINVAL),
                         (dict(out=264), EINVAL), (dict(ws=128), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
                         (dict(parent=256, rows=65, max_rows=65), ESHAPE), (dict(heads=4 << 20, qs=1 << 28), ESHAPE)]:
        a = dict(good, **change)
        rc = L.csd_paged_attention(ref, a["layer"], a["start"], a["pos"], a["parent"], a["B"], a["rows"], a["max_rows"], a["q"], a["qs"], a["heads"],
                                   a["dtype"], a["scale"], a["out"], a["ws"], None)
        assert rc == code, change
    assert L.csd_paged_attention(ref, 0, 256, 256, None, 1, 0, 1, None, 0, 8, 1, 0.125, None, None, None) == 0


def test_commit_refuses_what_it_cannot_do(L):
    ref, keep = _pool()
    assert L.csd_paged_commit(ref, None, 256, 256, 1, 8, None) == ENULL
    assert L.csd_paged_commit(ref, 256, None, 256, 1, 8, None) == ENULL
    assert L.csd_paged_commit(ref, 256, 256, None, 1, 8, None) == ENULL
    assert L.csd_paged_commit(ref, 256, 256, 256, 0, 8, None) == EINVAL
    assert L.csd_paged_commit(ref, 256, 256, 256, 1, 0, None) == EINVAL
    assert L.csd_paged_commit(ref, 256, 256, 256, 1, 65, None) == ESHAPE


def test_binding_refuses_host_tensors_and_wrong_pools():
    import paper_2312_11462_amd as P
    k = torch.zeros(1, 2, 4, 16, 64)
    with pytest.raises(ValueError):
        P.PagedKv(k, k.clone())                                        # host memory
    with pytest.raises(ValueError):
        P.PagedKv(k, k[:, :1])
    with pytest.raises(ValueError):
        P.PagedKv(k.half(), k.half())
    with pytest.raises(ValueError):
        P.PagedKv(k, k, k_scale=torch.zeros(1, 2, 4, 16, dtype=torch.uint8))
    with pytest.raises(ValueError):
        P.PagedKv(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn))


def test_attention_over_trees_goes_by_the_rows_there_are(L):
    """max_rows is cut to the rows of the call before it is held against the 64 rows of a tree (the output's address is refused behind that)."""
    ref, keep = _pool()
    for rows, most, code in ((40, 100, EINVAL), (64, 65, EINVAL), (65, 64, EINVAL), (65, 65, ESHAPE), (100, 1 << 20, ESHAPE)):
        assert L.csd_paged_attention(ref, 0, 256, 256, 256, 1, rows, most, 256, 512, 8, 1, 0.125, 264, 256, None) == code, (rows, most)
    assert L.csd_paged_attention(ref, 0, 256, 256, 256, 1, 0, 100, None, 0, 8, 1, 0.125, None, None, None) == 0


def test_capture_of_a_stream_needs_a_place_for_the_answer(L):
    assert L.csd_stream_capture(None, None) == ENULL


def test_a_workspace_is_asked_for_where_it_is_used(L):
    """(the queries' distance is refused behind that)"""
    for pool, heads_of, dtype, code in ((2, 64, 1, ENULL), (1, 128, 1, ENULL), (0, 64, 1, EINVAL), (1, 64, 0, EINVAL), (2, 80, 1, EINVAL), (0, 16, 0, EINVAL)):
        ref, keep = _pool(dtype=pool, head_dim=heads_of)
        assert L.csd_paged_attention(ref, 0, 256, 256, None, 1, 4, 4, 256, 4, 8, dtype, 0.125, 256, None, None) == code, (pool, heads_of, dtype)
