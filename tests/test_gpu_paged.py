"""The paged KV cache on the GPU against the plain form in 64 bits (oracle/paged.py).

Bounds.  A value rounded to a type is off by at most u = eps / 2 of itself (bf16 2^-8, fp32 2^-24).  An attention output is sum p v with
weights off by (1 + u_p) exp(e): u_p = 2^-8 where the weights are rounded to bf16 on their way into the matrix cores, and e the error of a
score, at most (D + 4) 2^-24 scale sum |q k| from the fp32 product, plus 2^-21 for the exponential and its argument (|x| <= 64 in steps of
2^-24 times the bits, two roundings) and n 2^-24 for the sums over n keys.  So
|out - exact| <= u_out |exact| + 2 (u_p + e) sum p |v|, the factor 2 for the sum of weights in the denominator.
"""
import math

import numpy as np
import pytest
import torch

from oracle import paged as O

pytestmark = pytest.mark.gpu

TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2312_11462_amd as P
    P.lib()


class Paged:
    """A cache on the GPU, and the values it holds as float64 on the host."""

    def __init__(self, cache, rows, cached, new, kv_heads=2, group=1, d=64, page=16, layers=1, seed=0, spare=3, width=0, poison=True):
        import paper_2312_11462_amd as P
        self.rng = np.random.default_rng(seed)
        self.cache, self.rows, self.cached, self.new = cache, rows, list(cached), list(new)
        self.kv_heads, self.group, self.d, self.page, self.layers = kv_heads, group, d, page, layers
        need = [-(-(t + m) // page) for t, m in zip(cached, new)]
        self.n_pages = sum(need) + spare
        order = self.rng.permutation(self.n_pages)
        self.table = np.full((len(cached), max(max(need), 1) + width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.total = int(self.start[-1])
        shape = (layers, self.n_pages, kv_heads, page, d)
        # places that nobody wrote hold NaN
        if cache == "fp8":
            self.k = torch.full(shape, 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            self.v = self.k.view(torch.uint8).clone().view(torch.float8_e4m3fn)
            self.ks = torch.full(shape[:-1], 200, dtype=torch.uint8, device="cuda")
            self.vs = self.ks.clone()
        else:
            fill = float("nan") if poison else 0.0
            self.k = torch.full(shape, fill, dtype=TORCH[cache], device="cuda")
            self.v = self.k.clone()
            self.ks = self.vs = None
        self.kv = P.PagedKv(self.k, self.v, self.ks, self.vs)
        self.dev = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (self.table, self.start, np.array(cached, dtype=np.int32))]

    def values(self, pool, scale):
        if scale is None:
            return pool.double().cpu().numpy()
        x = pool.view(torch.uint8).cpu().view(torch.float8_e4m3fn).double().numpy()
        return x * np.exp2(scale.cpu().numpy().astype(np.float64) - 127)[..., None]

    def random_rows(self, n, heads=None, loud=True):
        x = self.rng.standard_normal((n, heads or self.kv_heads, self.d))
        if loud:
            x[:, :, self.rng.integers(self.d)] *= 5
        return torch.tensor(x, dtype=torch.float32).to(TORCH[self.rows]).cuda()

    def fill(self, layer=0):
        """Writes every row, cached and new, with one call; returns the dense rows."""
        whole = [t + m for t, m in zip(self.cached, self.new)]
        start = torch.tensor(np.concatenate([[0], np.cumsum(whole)]), dtype=torch.int32, device="cuda")
        k, v = self.random_rows(sum(whole)), self.random_rows(sum(whole), loud=False)
        self.kv.write(layer, self.dev[0], start, torch.zeros(len(whole), dtype=torch.int32, device="cuda"), k, v)
        return k, v

    def attend(self, q, scale, max_rows=None, parent=None, layer=0, **kw):
        up = torch.tensor(parent, dtype=torch.int32, device="cuda") if parent is not None else None
        return self.kv.attention(layer, *self.dev, q, scale, max_rows, parent=up, **kw)

    def check(self, out, q, scale, parent=None, layer=0, start=None, cached=None):
        start, cached = self.start if start is None else start, self.cached if cached is None else cached
        k, v = self.values(self.k, self.ks)[layer], self.values(self.v, self.vs)[layer]
        qq = q.double().cpu().numpy()
        want = O.attention(k, v, self.table, start, cached, qq, scale, parent)
        size = O.attention(k, np.abs(v), self.table, start, cached, qq, scale, parent)
        n = max(t + m for t, m in zip(self.cached, self.new))
        # sum |q k| of a score is at most |q| |k| (Cauchy-Schwarz)
        live = k[np.isfinite(k).all(-1)]
        dot = abs(scale) * np.sqrt((qq ** 2).sum(-1)).max(initial=0) * np.sqrt((live ** 2).sum(-1)).max(initial=0)
        e = (self.d + 4) * 2.0 ** -24 * dot + 2.0 ** -21 + n * 2.0 ** -24
        bf = self.rows == "bf16"
        tol = (2.0 ** -8 if bf else 2.0 ** -24) * np.abs(want) + 2 * ((2.0 ** -8 if bf else 0.0) + e) * size
        got = out.double().cpu().numpy()
        covered = np.zeros(len(got), dtype=bool)
        covered[start[0]:start[-1]] = True
        assert np.array_equal(np.isfinite(got[covered]), np.isfinite(want[covered]))
        fine = np.isfinite(want) & covered[:, None, None]
        err = np.abs(got - want)[fine]
        assert (err <= tol[fine]).all(), f"off by {(err / np.maximum(tol[fine], 1e-300)).max():.2f} times the bound, {err.max():.3g}"
        return want


TYPES = [("fp32", "fp32"), ("fp32", "bf16"), ("fp32", "fp8"), ("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "fp32")]


@pytest.mark.parametrize("d,kv_heads,page", [(8, 1, 16), (64, 3, 16), (80, 2, 32), (128, 8, 64), (256, 1, 128)])
@pytest.mark.parametrize("rows,cache", TYPES)
def test_rows_in_and_out(rows, cache, d, kv_heads, page):
    """Ragged sequences, one without rows, one over a page border; what is not written keeps its bytes."""
    c = Paged(cache, rows, [0, 5, page - 1, 3 * page, 2], [1, 0, 2, page + 3, 17], kv_heads=kv_heads, d=d, page=page, layers=2, seed=d)
    for x, s in ((c.k, c.ks), (c.v, c.vs)):
        x.view(torch.uint8).copy_(torch.randint(0, 100, x.view(torch.uint8).shape, dtype=torch.uint8))
        if s is not None:
            s.copy_(torch.randint(100, 150, s.shape, dtype=torch.uint8))
    before = [c.values(c.k, c.ks), c.values(c.v, c.vs)]
    k, v = c.random_rows(c.total), c.random_rows(c.total)
    special = c.total - 1
    k[special, 0] = 0
    v[special, 0, :3] = torch.tensor([1e30, -1e-30, 3e4])
    c.kv.write(1, *c.dev, k, v)
    where = O.places(c.start, c.cached, c.table, page, c.n_pages, c.total)
    for pool, scale, was, x in ((c.k, c.ks, before[0], k), (c.v, c.vs, before[1], v)):
        dense = x.double().cpu().numpy()
        if cache == "fp8":
            dense, byte = O.quantise(dense)
            bytes_ = scale.cpu().numpy()[1]
            assert all(np.array_equal(bytes_[page_, :, slot], byte[r]) for r, _, _, page_, slot in where)
        elif cache == "bf16":
            dense = x.float().cpu().to(torch.bfloat16).double().numpy()
        O.write(was[1], dense, where)
        assert np.array_equal(c.values(pool, scale), was)
    t = TORCH[rows]
    got = c.kv.read(1, *c.dev, c.total, dtype=t)
    for pool, scale, x in ((c.k, c.ks, got[0]), (c.v, c.vs, got[1])):
        want = O.read(c.values(pool, scale)[1], where, c.total)
        assert np.array_equal(x.double().cpu().numpy(), torch.tensor(want).to(t).double().numpy())


def test_quantised_rows_at_the_borders_of_the_type():
    """Rows whose maximum sits at a step of the scale, in fp32's subnormal range, or is zero; ties; NaN and infinities among the entries."""
    d = 64
    rows = []
    for top in (448.0, 448.00003, 224.0, 1.75, 1.7500001, 3.4e38, 1e-37, 1.2e-38, 1e-40, 0.0):
        x = np.linspace(-1, 1, d) * top
        x[3] = top
        rows.append(x)
    ties = np.arange(d) * 0.5 + 1.0625 * 2.0 ** (np.arange(d) % 8)           # halfway between two codes at several exponents
    ties[0] = 448.0
    rows.append(ties)
    for bad in (np.nan, np.inf, -np.inf):
        x = np.linspace(-3, 5, d)
        x[7] = bad
        rows.append(x)
    rows.append(np.full(d, np.nan))
    x = torch.tensor(np.stack(rows), dtype=torch.float32).cuda()[:, None].contiguous()
    n = x.shape[0]
    c = Paged("fp8", "fp32", [0], [n], kv_heads=1, d=d)
    c.kv.write(0, *c.dev, x, x.flip(0).contiguous())
    want, byte = O.quantise(x.double().cpu().numpy())
    where = O.places(c.start, c.cached, c.table, c.page, c.n_pages, n)
    pool, scales = c.values(c.k, c.ks)[0], c.ks.cpu().numpy()[0]
    for r, _, _, page, slot in where:
        assert np.array_equal(scales[page, :, slot], byte[r]), r
        assert np.array_equal(pool[page, :, slot], want[r], equal_nan=True), r
    # a row that is read and written again keeps its values
    k, v = c.kv.read(0, *c.dev, n)
    c.kv.write(0, *c.dev, k, v)
    again = c.values(c.k, c.ks)[0]
    for r, _, _, page, slot in where:
        assert np.array_equal(again[page, :, slot], want[r], equal_nan=True), r


def test_rows_without_a_place_and_rows_of_no_sequence():
    c = Paged("bf16", "bf16", [0, 10], [20, 30], kv_heads=2, d=64, page=16)
    c.table[0, 1] = -1                                    # given back
    c.table[1, 0] = c.n_pages                             # out of range
    c.table[1, 2] = 2 ** 31 - 1
    c.dev[0].copy_(torch.tensor(c.table))
    pad = 7
    start = torch.tensor([pad, pad + 20, pad + 50], dtype=torch.int32, device="cuda")
    c.start = start.cpu().numpy()
    k, v = c.random_rows(pad + 50 + pad), c.random_rows(pad + 50 + pad)
    before = c.values(c.k, None)
    c.kv.write(0, c.dev[0], start, c.dev[2], k, v)
    where = O.places(c.start, c.cached, c.table, 16, c.n_pages, 10 ** 9)
    O.write(before[0], k.double().cpu().numpy(), where)
    assert np.array_equal(c.values(c.k, None), before, equal_nan=True)
    out = [torch.full((pad + 50 + pad, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    c.kv.read(0, c.dev[0], start, c.dev[2], pad + 50 + pad, out=out)
    want = O.read(before[0], where, pad + 50 + pad)
    want[:pad] = want[pad + 50:] = 9.0
    assert np.array_equal(out[0].double().cpu().numpy(), want)
    # rows past the end of the table
    short = c.dev[0][:, :1].contiguous()
    c.kv.read(0, short, start, c.dev[2], pad + 50 + pad, out=out)
    assert (out[0][pad + 16:pad + 20] == 0).all() and (out[0][pad + 26:pad + 50] == 0).all()


@pytest.mark.parametrize("rows,cache", [("bf16", "fp8"), ("fp32", "fp32")])
def test_rows_of_thousands_of_sequences(rows, cache):
    """None, one or a few each; in, out, and as single tokens attended."""
    rng = np.random.default_rng(3)
    new = rng.choice([0, 0, 1, 1, 1, 3, 20], 9001)
    new[:70], new[4200:4400] = 0, 0                                    # (whole groups of sequences without rows)
    c = Paged(cache, rows, rng.integers(0, 5, 9001), new, kv_heads=1, d=64, seed=13)
    k, v = c.random_rows(c.total), c.random_rows(c.total)
    c.kv.write(0, *c.dev, k, v)
    got = c.kv.read(0, *c.dev, c.total, dtype=TORCH[rows])
    for x, y in zip((k, v), got):
        want = O.quantise(x.double().cpu().numpy())[0] if cache == "fp8" else x.double().cpu().numpy()
        assert np.array_equal(y.double().cpu().numpy(), want)
    c.fill()
    q = c.random_rows(c.total, 2)
    c.check(c.attend(q, 0.125, 20), q, 0.125)


HEADS = [(1, 1), (2, 4), (8, 1), (1, 8), (4, 3)]


@pytest.mark.parametrize("rows,cache,d", [("fp32", "fp32", 16), ("fp32", "fp32", 64), ("fp32", "bf16", 128), ("fp32", "fp8", 64), ("bf16", "bf16", 64), ("bf16", "bf16", 128),
                                          ("bf16", "fp8", 64), ("bf16", "fp8", 128), ("bf16", "bf16", 80), ("bf16", "fp8", 256), ("bf16", "fp32", 64)])
@pytest.mark.parametrize("kv_heads,group", HEADS)
def test_attention_of_small_batches(rows, cache, d, kv_heads, group):
    """Single tokens, blocks and short chunks of one batch, at lengths around tiles and pages; a sequence without rows; an empty cache."""
    for page, new in ((16, [1, 1, 1, 1, 1, 1, 1, 1]), (32, [5, 0, 1, 5, 2, 5, 5, 4]), (16, [17, 1, 16, 0, 33, 3, 15, 8])):
        c = Paged(cache, rows, [0, 7, 31, 32, 33, 63, 127, 200], new, kv_heads=kv_heads, group=group, d=d, page=page, seed=page + d)
        c.fill()
        q = c.random_rows(c.total, kv_heads * group)
        out = c.attend(q, d ** -0.5, max(new))
        c.check(out, q, d ** -0.5)
        c.check(c.attend(q, d ** -0.5), q, d ** -0.5)        # another bound on the rows may take another kernel: the same limits, not the same bits


@pytest.mark.parametrize("rows,cache,d,kv_heads,group", [("bf16", "bf16", 128, 2, 4), ("bf16", "fp8", 128, 2, 2), ("bf16", "bf16", 64, 3, 1), ("bf16", "fp8", 64, 1, 8), ("fp32", "fp32", 32, 2, 2)])
@pytest.mark.parametrize("cached,new", [([0], [129]), ([77], [200]), ([0, 300, 5], [64, 65, 1]), ([1000], [70]), ([511, 2], [1, 257]), ([3, 0, 0], [300, 1, 0])])
def test_attention_of_chunks(rows, cache, d, kv_heads, group, cached, new):
    c = Paged(cache, rows, cached, new, kv_heads=kv_heads, group=group, d=d, page=64, seed=d + len(new))
    c.fill()
    q = c.random_rows(c.total, kv_heads * group)
    c.check(c.attend(q, d ** -0.5, max(new)), q, d ** -0.5)


@pytest.mark.parametrize("rows,cache,d,new", [("bf16", "bf16", 128, 1), ("bf16", "fp8", 128, 5), ("bf16", "bf16", 64, 1), ("bf16", "fp8", 64, 9), ("fp32", "fp32", 64, 2), ("bf16", "bf16", 128, 40)])
def test_attention_of_long_caches(rows, cache, d, new):
    """The work of a sequence is split over its keys and joined."""
    c = Paged(cache, rows, [9001, 3, 4097, 0], [new] * 4, kv_heads=2, group=2, d=d, page=16, seed=new)
    c.fill()
    q = c.random_rows(c.total, 4)
    out = c.attend(q, d ** -0.5, new)
    c.check(out, q, d ** -0.5)
    for _ in range(3):
        assert torch.equal(c.attend(q, d ** -0.5, new), out)           # sums in one order, and a workspace that is as it was


def test_attention_of_many_sequences():
    n = 150                                                             # more than a wave looks at in one go
    rng = np.random.default_rng(1)
    c = Paged("bf16", "bf16", rng.integers(0, 90, n), rng.integers(0, 4, n), kv_heads=1, group=2, d=64, seed=2)
    c.fill()
    q = c.random_rows(c.total, 2)
    c.check(c.attend(q, 0.125, 3), q, 0.125)
    c.check(c.attend(q, 0.125), q, 0.125)


SPREAD = [("fp32", "fp32", 32), ("bf16", "bf16", 128), ("bf16", "fp8", 64), ("bf16", "bf16", 80)]


@pytest.mark.parametrize("rows,cache,d", SPREAD)
@pytest.mark.parametrize("m,group", [(2, 1), (9, 1), (41, 1), (64, 1), (9, 4), (33, 2)])
def test_attention_over_trees(rows, cache, d, m, group):
    rng = np.random.default_rng(m)
    c = Paged(cache, rows, [0, 65, 130], [m] * 3, kv_heads=2, group=group, d=d, seed=m)
    c.fill()
    parent = np.concatenate([[int(rng.integers(max(0, i - 9), i)) if i else -1 for i in range(m)] for _ in range(3)]).astype(np.int32)
    q = c.random_rows(c.total, 2 * group)
    c.check(c.attend(q, d ** -0.5, m, parent), q, d ** -0.5, parent)
    chain = np.concatenate([np.arange(m) - 1] * 3).astype(np.int32)
    plain = c.attend(q, d ** -0.5, m)
    c.check(c.attend(q, d ** -0.5, m, chain), q, d ** -0.5)
    wild = parent.copy()
    wild[m // 2] = m                                                    # outside [0, i): read as 0
    wild[-1] = -7
    c.check(c.attend(q, d ** -0.5, m, wild), q, d ** -0.5, wild)
    assert torch.equal(plain, c.attend(q, d ** -0.5, m))


@pytest.mark.parametrize("rows,cache,d", SPREAD)
@pytest.mark.parametrize("m", [1, 3, 50])
def test_pages_that_were_given_back_and_rows_with_nothing_to_attend(rows, cache, d, m):
    c = Paged(cache, rows, [100, 200, 5, 0], [m, m, m, 1], kv_heads=2, group=2, d=d, seed=m)
    c.fill()
    c.table[0, 2:4] = -1
    c.table[1, 0], c.table[1, 5] = c.n_pages, -5
    c.table[2] = -1                                                     # nothing left
    c.dev[0].copy_(torch.tensor(c.table))
    q = c.random_rows(c.total, 4)
    out = c.attend(q, d ** -0.5, m)
    c.check(out, q, d ** -0.5)
    assert (out[2 * m:3 * m] == 0).all()


@pytest.mark.parametrize("rows,cache,d", SPREAD)
@pytest.mark.parametrize("m,tree", [(2, False), (16, False), (40, False), (70, False), (40, True)])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_reach_only_the_rows_that_attend_them(rows, cache, d, m, tree, what):
    """A later token of the block, or a row beside this one in the tree, has such keys or values."""
    c = Paged(cache, rows, [37, 0], [m, m], kv_heads=2, group=2, d=d, seed=m)
    k, v = c.fill()
    bad = m // 2
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    kr, vr = c.random_rows(1), c.random_rows(1)
    vr[0, 1, d // 3] = what
    c.kv.write(0, c.dev[0][:1].contiguous(), one, torch.tensor([37 + bad], dtype=torch.int32, device="cuda"), kr, vr)
    kr, vr = c.random_rows(1), c.random_rows(1)
    kr[0, 0, 1] = what
    c.kv.write(0, c.dev[0][1:].contiguous(), one, torch.tensor([bad], dtype=torch.int32, device="cuda"), kr, vr)
    parent = np.concatenate([[-1] + [0] * (m - 1)] * 2).astype(np.int32) if tree else None
    q = c.random_rows(c.total, 4).abs()
    out = c.attend(q, d ** -0.5, m, parent).float().cpu()
    clean_rows = [i for i in range(m) if (i != bad if tree else i < bad)]
    assert torch.isfinite(out[clean_rows]).all() and torch.isfinite(out[[m + i for i in clean_rows]]).all()
    # the values' feature of the second key-value head, in the rows that attend the bad one: as the formula has it
    assert not torch.isfinite(out[bad, 2:, d // 3]).any()
    rest = torch.ones(d, dtype=torch.bool)
    rest[d // 3] = False
    assert torch.isfinite(out[bad, 2:, rest]).all() and torch.isfinite(out[bad, :2]).all()
    kk, vv = c.values(c.k, c.ks)[0], c.values(c.v, c.vs)[0]
    with np.errstate(invalid="ignore"):
        want = O.attention(kk, vv, c.table, c.start, c.cached, q.double().cpu().numpy(), d ** -0.5, parent)
    ok = np.isfinite(want)
    assert np.allclose(out.double().numpy()[ok], want[ok], rtol=0.05, atol=0.05)


@pytest.mark.parametrize("rows,cache,d,m", [("bf16", "bf16", 128, 3), ("bf16", "fp8", 64, 60), ("fp32", "fp32", 64, 3)])
def test_large_scores(rows, cache, d, m):
    """Scores of several hundred, one key that takes all the weight, and a later key that takes it over."""
    c = Paged(cache, rows, [300], [m], kv_heads=1, group=2, d=d)
    c.fill()
    q = c.random_rows(m, 2)
    c.check(c.attend(q, 8.0, m), q, 8.0)
    c.check(c.attend(q, -3.0, m), q, -3.0)
    c.check(c.attend(q, 0.0, m), q, 0.0)


@pytest.mark.parametrize("rows,cache,d,m", [("bf16", "fp8", 128, 4), ("bf16", "bf16", 64, 100), ("fp32", "fp32", 16, 3)])
def test_rows_inside_a_wider_buffer_and_padded_batches(rows, cache, d, m):
    """Queries, keys and values as slices of one projection's output; rows behind the last sequence are left as they were."""
    c = Paged(cache, rows, [40, 11], [m, m], kv_heads=2, group=2, d=d)
    c.fill()
    pad = 5
    fused = torch.randn(2 * m + pad, (4 + 2 + 2) * d + 8, device="cuda").to(TORCH[rows])
    q = fused[:, :4 * d].view(2 * m + pad, 4, d)
    k = fused[:, 4 * d:6 * d].view(2 * m + pad, 2, d)
    v = fused[:, 6 * d:8 * d].view(2 * m + pad, 2, d)
    c.kv.write(0, *c.dev, k, v)
    out = torch.full((2 * m + pad, 4, d), 7.0, dtype=TORCH[rows], device="cuda")
    got = c.attend(q, d ** -0.5, m, out=out)
    assert got is out and (out[2 * m:] == 7).all()
    c.check(out[:2 * m], q[:2 * m], d ** -0.5)
    back = c.kv.read(0, *c.dev, 2 * m + pad, out=(fused[:, 4 * d:6 * d].view(2 * m + pad, 2, d), fused[:, 6 * d:8 * d].view(2 * m + pad, 2, d)))
    assert torch.equal(back[0][2 * m:], k[2 * m:])


@pytest.mark.parametrize("cache", ["fp32", "bf16", "fp8"])
def test_commit_of_a_trees_path(cache):
    m, page = 41, 16
    c = Paged(cache, "fp32" if cache == "fp32" else "bf16", [0, 33, 15, 7, 9], [m] * 5, kv_heads=3, d=64, page=page, layers=3, seed=4)
    for layer in range(3):
        c.fill(layer)
    path = np.full((5, m), -1, dtype=np.int32)
    kept = np.array([4, 0, 40, 3, 60], dtype=np.int32)
    path[0, :4] = [1, 9, 17, 40]
    path[2, :40] = np.arange(1, 41)                       # everything is where it belongs
    path[3, :3] = [2, 5, 5]                               # not increasing: cut at the third
    path[4, :6] = [3, 4, 5, 6, 7, 41]                     # out of the block: cut at the sixth
    c.table[0, 1] = -1                                    # rows 16 .. 31 of the first sequence have no place
    c.dev[0].copy_(torch.tensor(c.table))
    pools = [c.values(c.k, c.ks), c.values(c.v, c.vs)]
    for pool in pools:
        O.commit(pool, c.table, c.cached, path, kept)
    c.kv.commit(c.dev[0], c.dev[2], torch.tensor(path).cuda(), torch.tensor(kept).cuda())
    assert np.array_equal(c.values(c.k, c.ks), pools[0], equal_nan=True) and np.array_equal(c.values(c.v, c.vs), pools[1], equal_nan=True)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_a_review_over_pages_write_attend_commit_and_the_next_block(cache):
    """As a decoding loop does it: the rows of a tree are written and attended, a path is kept, the next block sees it as plain rows."""
    m, d = 9, 128
    c = Paged(cache, "bf16", [50, 17], [m, m], kv_heads=2, group=2, d=d, layers=2, width=1, seed=8)
    c.fill(0)
    c.fill(1)
    k, v = c.random_rows(2 * m), c.random_rows(2 * m)
    parent = np.array([-1, 0, 0, 1, 1, 2, 3, 4, 7] * 2, dtype=np.int32)
    path = np.array([[2, 5, 0, 0, 0, 0, 0, 0, 0], [1, 4, 7, 8, 0, 0, 0, 0, 0]], dtype=np.int32)
    kept = np.array([2, 4], dtype=np.int32)
    q = c.random_rows(2 * m, 4)
    for layer in range(2):
        c.kv.write(layer, *c.dev, k, v)
        c.check(c.attend(q, 0.1, m, parent, layer=layer), q, 0.1, parent, layer=layer)
    tree = c.attend(q, 0.1, m, parent)
    c.kv.commit(c.dev[0], c.dev[2], torch.tensor(path).cuda(), torch.tensor(kept).cuda())
    # the kept rows as a plain block of their own, with the same queries: the same outputs up to rounding
    rows = np.concatenate([[0] + list(path[0, :2]), [0] + list(path[1, :4])])
    rows[3:] += m
    start = torch.tensor([0, 3, 8], dtype=torch.int32, device="cuda")
    block = c.kv.attention(0, c.dev[0], start, c.dev[2], q[rows].contiguous(), 0.1, 5)
    c.check(block, q[rows], 0.1, start=np.array([0, 3, 8]))
    size = tree.float().abs().max()
    assert ((block.float() - tree[torch.tensor(rows).cuda()].float()).abs() <= 2.0 ** -6 * size).all()


@pytest.mark.parametrize("m", [1, 6, 80])
def test_captured_calls_replay_to_the_eager_result(m):
    c = Paged("fp8", "bf16", [600, 0, 1500], [m] * 3, kv_heads=2, group=2, d=128, width=2, seed=m)
    c.fill()
    q, k, v = c.random_rows(3 * m, 4), c.random_rows(3 * m), c.random_rows(3 * m)
    out = torch.zeros_like(q)

    def step():
        c.kv.write(0, *c.dev, k, v)
        c.kv.attention(0, *c.dev, q, 0.09, m, out=out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        q.copy_(c.random_rows(3 * m, 4))
        k.copy_(c.random_rows(3 * m))
        c.dev[2].copy_(torch.tensor([600 - rep, 2 * rep, 1500 - 300 * rep]))
        step()
        torch.cuda.synchronize()
        want = out.clone()
        out.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)), rep      # bits: the second sequence meets rows that nobody wrote, NaN


def test_calls_on_another_stream_follow_that_stream():
    c = Paged("bf16", "bf16", [700], [3], kv_heads=2, group=2, d=128)
    c.fill()
    q = c.random_rows(3, 4)
    want = c.attend(q, 0.1, 3)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = torch.zeros_like(q)
        for _ in range(20):
            late.copy_(q)                                  # in order on that stream
        got = c.attend(late, 0.1, 3)
    side.synchronize()
    assert torch.equal(got, want)


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB, the rows at its end."""
    import paper_2312_11462_amd as P
    heads, page, d = 8, 128, 128
    n = (1 << 32) // (heads * page * d) + 40               # codes of 2^32 bytes and some
    c = Paged("fp8", "bf16", [300], [3], kv_heads=heads, d=d, page=page)
    small = c.n_pages
    c.n_pages = n
    c.k = torch.empty((1, n, heads, page, d), dtype=torch.float8_e4m3fn, device="cuda")
    c.v = torch.empty_like(c.k)
    c.ks = torch.empty((1, n, heads, page), dtype=torch.uint8, device="cuda")
    c.vs = torch.empty_like(c.ks)
    for x in (c.k.view(torch.uint8), c.v.view(torch.uint8)):
        x.fill_(0x7F)
    c.kv = P.PagedKv(c.k, c.v, c.ks, c.vs)
    c.table[0, :3] = [n - 1, n - 7, n - 39]
    c.dev[0].copy_(torch.tensor(c.table))
    k, v = c.fill()
    back = c.kv.read(0, c.dev[0], torch.tensor([0, 303], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 303)
    want, _ = O.quantise(k.double().cpu().numpy())
    assert np.array_equal(back[0].double().cpu().numpy(), want)
    q = c.random_rows(3, heads)
    out = c.attend(q, 0.1, 3)
    # the same rows in a small pool give the same bits
    s = Paged("fp8", "bf16", [300], [3], kv_heads=heads, d=d, page=page)
    s.kv.write(0, s.dev[0], torch.tensor([0, 303], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), k, v)
    assert torch.equal(out, s.attend(q, 0.1, 3)) and small < n
    path = torch.full((1, 3), -1, dtype=torch.int32, device="cuda")
    path[0, 0] = 2
    for x in (c, s):
        x.kv.commit(x.dev[0], x.dev[2], path, torch.ones(1, dtype=torch.int32, device="cuda"))
    assert torch.equal(c.attend(q, 0.1, 3), s.attend(q, 0.1, 3))


def test_a_models_sequence_is_parked_in_the_pool_and_taken_back():
    """The rows of a model's dense cache go into pages (a bf16 pool keeps them exactly) and come back into another slot: the next review is the same
    to the bit.  Attention over the pages is the model's own, seen through its first layer."""
    import csd_inputs as I
    import paper_2312_11462_amd as P
    shape = I.ModelShape("park", 0, "bf16", 3, 256, 4, 64, 512, 1024)
    gm = P.Model(shape, I.make_weights(shape, 5, device="cuda", std=0.05), max_batch=2, max_seq=160, max_block=8)
    toks = I.token_ids(120, shape.vocab, 5, 1).cuda()
    n = 96
    for pos in range(0, n, 8):
        both = toks[None, pos:pos + 8].expand(2, 8).contiguous()
        gm.verify_block(both, torch.full((2,), pos, dtype=torch.int32, device="cuda"))
    block = toks[None, n:n + 5].expand(2, 5).contiguous()
    cl = torch.full((2,), n, dtype=torch.int32, device="cuda")
    want = gm.verify_block(block, cl)[0].clone()
    k = torch.zeros((3, 8, 4, 16, 64), dtype=torch.bfloat16, device="cuda")
    kv = P.PagedKv(k, torch.zeros_like(k))
    table = torch.tensor([[5, 0, 7, 2, 1, 6]], dtype=torch.int32, device="cuda")
    start, zero = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for layer in range(3):
        K, V = gm.kv_read(layer, 0, 0, n)
        kv.write(layer, table, start, zero, K.view(n, 4, 64), V.view(n, 4, 64))
    junk = torch.randn(n, 256, device="cuda")
    for layer in range(3):
        gm.kv_write(layer, 0, 0, junk, junk)
    assert not torch.equal(gm.verify_block(block, cl)[0], want)
    for layer in range(3):
        K, V = kv.read(layer, table, start, zero, n)
        gm.kv_write(layer, 0, 0, K.reshape(n, 256), V.reshape(n, 256))
    assert torch.equal(gm.verify_block(block, cl)[0], want)


@pytest.mark.parametrize("rows,cache,d,kv_heads,n", [("bf16", "fp8", 256, 17, 1931), ("fp32", "fp8", 64, 5, 26250), ("bf16", "bf16", 8, 33, 31801), ("bf16", "fp8", 80, 6, 10931)])
def test_many_rows_in_and_out(rows, cache, d, kv_heads, n):
    """So many that a wave takes several heads; head counts that are no multiple of these, row counts that end inside a wave."""
    c = Paged(cache, rows, [3, 0, 70], [n - 5, 0, 5], kv_heads=kv_heads, d=d, page=64, seed=d)
    c.table[0, 2] = -1
    c.dev[0].copy_(torch.tensor(c.table))
    k, v = c.random_rows(n), c.random_rows(n)
    before = [c.values(c.k, c.ks)[0], c.values(c.v, c.vs)[0]]
    c.kv.write(0, *c.dev, k, v)
    where = O.places(c.start, c.cached, c.table, c.page, c.n_pages, n)
    for pool, scale, was, x in ((c.k, c.ks, before[0], k), (c.v, c.vs, before[1], v)):
        dense = x.double().cpu().numpy()
        O.write(was, O.quantise(dense)[0] if cache == "fp8" else dense, where)
        got = c.values(pool, scale)[0]
        used = np.unique([page for _, _, _, page, _ in where if page >= 0])
        if cache == "fp8":                                              # (places that nobody wrote: NaN whatever their scale)
            assert np.array_equal(got[used], was[used], equal_nan=True)
        else:
            assert np.array_equal(got, was, equal_nan=True)
    back = c.kv.read(0, *c.dev, n, dtype=TORCH[rows])
    for was, x in zip(before, back):
        assert np.array_equal(x.double().cpu().numpy(), torch.tensor(O.read(was, where, n)).to(TORCH[rows]).double().numpy())


@pytest.mark.parametrize("rows,cache,d", [("bf16", "bf16", 64), ("bf16", "fp8", 128), ("bf16", "fp8", 64), ("bf16", "bf16", 128)])
def test_attention_of_more_sequences_than_share_their_keys(rows, cache, d):
    """More than 512 sequences; many row tiles of short blocks, and of longer ones; single tokens beside them, lengths of every kind."""
    rng = np.random.default_rng(d)
    cached, new = rng.integers(0, 70, 530), rng.choice([0, 1, 5, 9], 530)
    cached[7], new[7] = 300, 41
    c = Paged(cache, rows, cached, new, kv_heads=1, group=8, d=d, seed=5)
    c.fill()
    q = c.random_rows(c.total, 8)
    c.check(c.attend(q, d ** -0.5, 41), q, d ** -0.5)
    c = Paged(cache, rows, rng.integers(0, 40, 140), np.append(rng.integers(33, 40, 139), 150), kv_heads=8, d=d, seed=6)
    c.fill()
    q = c.random_rows(c.total, 8)
    c.check(c.attend(q, d ** -0.5, 150), q, d ** -0.5)
    c = Paged(cache, rows, [40, 0, 9], [200, 1, 130], kv_heads=96, group=4, d=d, page=32, seed=7)
    c.fill()
    q = c.random_rows(c.total, 384)
    c.check(c.attend(q, d ** -0.5, 200), q, d ** -0.5)


@pytest.mark.parametrize("rows,cache,d", [("bf16", "bf16", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 64), ("bf16", "fp8", 128)])
def test_chunks_far_apart_in_a_large_batch(rows, cache, d):
    """Hundreds of single tokens, and sequences without rows, between the few sequences of many rows."""
    rng = np.random.default_rng(d)
    cached, new = rng.integers(0, 60, 1300), (rng.random(1300) < 0.7).astype(int)
    for b, t, m in ((5, 400, 70), (300, 0, 33), (640, 1000, 129), (1299, 10, 17)):
        cached[b], new[b] = t, m
    c = Paged(cache, rows, cached, new, kv_heads=2, d=d, seed=12)
    c.fill()
    q = c.random_rows(c.total, 2)
    c.check(c.attend(q, d ** -0.5, 129), q, d ** -0.5)


FULL = [("bf16", "bf16", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 64), ("bf16", "fp8", 128)]
MORE = 520                                                              # short sequences beside the ones at hand: too many for the keys to be shared out


@pytest.mark.parametrize("rows,cache,d", FULL)
@pytest.mark.parametrize("page", [16, 128])
def test_chunks_beside_many_short_ones(rows, cache, d, page):
    """Whole workgroups of rows: lengths of one tile to fifty, row counts around a wave and a workgroup, negative scales, rows in a wider buffer."""
    cached, new = [3000, 3, 1500, 1023, 64, 0, 447, 512], [130, 129, 20, 64, 1, 257, 65, 16]
    c = Paged(cache, rows, cached + [0] * MORE, new + [9] * MORE, kv_heads=2, group=2, d=d, page=page, seed=page)
    c.fill()
    wide = torch.randn(c.total, 4 * d + 24, device="cuda").to(TORCH[rows])
    q = wide[:, 8:8 + 4 * d].unflatten(1, (4, d))
    out = c.attend(q, d ** -0.5, 257)
    c.check(out, q, d ** -0.5)
    for _ in range(3):
        assert torch.equal(c.attend(q, d ** -0.5, 257), out)
    c.check(c.attend(q, -0.3, 257), q, -0.3)


@pytest.mark.parametrize("rows,cache,d", FULL)
@pytest.mark.parametrize("m", [33, 41, 64])
def test_trees_beside_many_short_ones(rows, cache, d, m):
    rng = np.random.default_rng(m)
    n = 3
    c = Paged(cache, rows, [0, 601, 130] + [0] * MORE, [m] * n + [5] * MORE, kv_heads=2, group=4, d=d, seed=m)
    c.fill()
    c.table[1, 3:6] = -1
    c.dev[0].copy_(torch.tensor(c.table))
    parent = np.concatenate([[int(rng.integers(max(0, i - 9), i)) if i else -1 for i in range(m)] for _ in range(n)] + [[-1, 0, 0, 1, 3]] * MORE).astype(np.int32)
    q = c.random_rows(c.total, 8)
    c.check(c.attend(q, d ** -0.5, m, parent), q, d ** -0.5, parent)
    c.check(c.attend(q, 0.0, m, parent), q, 0.0, parent)


@pytest.mark.parametrize("rows,cache,d", FULL)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_beside_many_short_ones(rows, cache, d, tree, what):
    """In front of the block, in it, and behind it on the last page; a sequence whose pages are all gone."""
    m = 50
    c = Paged(cache, rows, [700, 0, 90] + [0] * MORE, [m, m, m] + [9] * MORE, kv_heads=2, group=2, d=d, seed=m)
    c.fill()
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for b, at, entry in ((0, 730, 3), (1, 20, d - 1)):
        kr, vr = c.random_rows(1), c.random_rows(1)
        vr[0, 1, entry] = what
        c.kv.write(0, c.dev[0][b:b + 1].contiguous(), one, torch.tensor([at], dtype=torch.int32, device="cuda"), kr, vr)
    kr, vr = c.random_rows(1), c.random_rows(1)
    kr[0, 0, 1] = what                                                  # a key
    c.kv.write(0, c.dev[0][0:1].contiguous(), one, torch.tensor([745], dtype=torch.int32, device="cuda"), kr, vr)
    c.table[2] = -1
    c.dev[0].copy_(torch.tensor(c.table))
    parent = np.concatenate([[-1] + [i // 2 for i in range(m - 1)]] * 3 + [np.arange(9) - 1] * MORE).astype(np.int32) if tree else None
    q = c.random_rows(c.total, 4)
    with np.errstate(invalid="ignore"):
        want = c.check(c.attend(q, 0.2, m, parent), q, 0.2, parent)
    assert (want[2 * m:3 * m] == 0).all() and np.isfinite(want[:10]).all() and not np.isfinite(want).all()


@pytest.mark.parametrize("rows,cache,d", SPREAD + [("bf16", "bf16", 64), ("bf16", "fp8", 128)])
@pytest.mark.parametrize("most,others", [(1, 0), (5, 0), (40, 0), (40, MORE)])
def test_sequences_longer_than_said_are_cut(rows, cache, d, most, others):
    """Their first rows are what they are, the others stay as they were."""
    new = [60, 3, 41, 1] + [9] * others
    c = Paged(cache, rows, [100, 0, 31, 7] + [0] * others, new, kv_heads=2, group=2, d=d, seed=most)
    c.fill()
    q = c.random_rows(c.total, 4)
    out = torch.full_like(q, 3.0)
    c.attend(q, d ** -0.5, most, out=out)
    kept = np.concatenate([np.arange(m) < most for m in new])
    assert (out[torch.tensor(~kept).cuda()] == 3).all()
    whole = c.attend(q, d ** -0.5, 60)
    c.check(whole, q, d ** -0.5)
    whole[torch.tensor(kept).cuda()] = out[torch.tensor(kept).cuda()]
    c.check(whole, q, d ** -0.5)


@pytest.mark.parametrize("rows,cache,d", SPREAD + [("bf16", "bf16", 64), ("bf16", "fp8", 128)])
def test_attention_of_blocks_of_every_size_in_one_batch(rows, cache, d):
    """1 .. 70 rows times two query heads: the sizes where one way of doing it ends and another begins; rows in front of the first sequence and behind
    the last stay as they are."""
    new = [1, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 70, 1]
    c = Paged(cache, rows, [40 * i % 330 for i in range(len(new))], new, kv_heads=2, group=2, d=d, seed=9)
    c.fill()
    lead, tail = 3, 4
    start = c.start + lead
    c.dev[1].copy_(torch.tensor(start))
    q = c.random_rows(c.total + lead + tail, 4)
    out = torch.full_like(q, 5.0)
    c.attend(q, d ** -0.5, 70, out=out)
    c.check(out, q, d ** -0.5, start=start)
    assert (out[:lead] == 5).all() and (out[-tail:] == 5).all()


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_a_million_cached_positions(cache):
    """A share of the keys is longer than the pages that are held at a time; as a single token, and as a block of more rows."""
    n = 1_100_000
    c = Paged(cache, "bf16", [n], [1], kv_heads=1, d=64, page=16)
    k, v = c.fill()
    # feature f is large in the f-th of 64 stretches of the keys: a stretch left out, or taken twice, shows
    v = (v * 0.1).to(torch.bfloat16) + 8 * torch.nn.functional.one_hot(torch.arange(n + 1, device="cuda") * 64 // (n + 1), 64).to(torch.bfloat16)[:, None]
    c.kv.write(0, c.dev[0], torch.tensor([0, n + 1], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), k, v)
    q = c.random_rows(1, 1)
    whole = q * 0.125                                                   # (exact: a power of two)
    x = (k[:, 0].double() if cache == "bf16" else torch.tensor(O.quantise(k[:, 0].double().cpu().numpy())[0]).cuda()) @ whole[0, 0].double()
    vv = v[:, 0].double() if cache == "bf16" else torch.tensor(O.quantise(v[:, 0].double().cpu().numpy())[0]).cuda()
    w = torch.softmax(x, 0)
    want, size = w @ vv, w @ vv.abs()
    dot = whole.double().norm() * k.double().norm(dim=-1).max()
    # as in the head of this file; no sum runs over more than a tenth of the keys before it is joined with the others
    tol = 2.0 ** -8 * want.abs() + 2 * (2.0 ** -8 + 68 * 2.0 ** -24 * dot + 2.0 ** -21 + n / 10 * 2.0 ** -24) * size
    got = c.attend(q, 0.125, 1)
    assert ((got[0, 0].double() - want).abs() <= tol).all()
    # a block of 40 rows that ends there, row 39 the same query
    c.dev[1].copy_(torch.tensor([0, 40]))
    c.dev[2].copy_(torch.tensor([n - 39]))
    block = c.random_rows(40, 1)
    block[39] = q[0]
    got = c.attend(block, 0.125, 40)
    assert ((got[39, 0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("rows,cache,d", SPREAD + [("bf16", "bf16", 64), ("bf16", "fp8", 128)])
@pytest.mark.parametrize("m", [3, 40])
def test_a_scale_of_zero_weighs_all_alike(rows, cache, d, m):
    """However large the products of queries and keys are."""
    c = Paged(cache, rows, [70, 0], [m, m], kv_heads=2, group=2, d=d, seed=m)
    k, v = c.fill()
    start = torch.tensor([0, 70 + m, 70 + 2 * m], dtype=torch.int32, device="cuda")
    c.kv.write(0, c.dev[0], start, torch.zeros(2, dtype=torch.int32, device="cuda"), k * 2.0 ** 56, v)
    q = c.random_rows(2 * m, 4) * 2.0 ** 56
    c.check(c.attend(q, 0.0, m), q, 0.0)


@pytest.mark.parametrize("rows,cache,d,m", [("bf16", "bf16", 128, 2), ("bf16", "bf16", 64, 40), ("bf16", "fp8", 64, 12), ("bf16", "fp8", 128, 40), ("fp32", "fp32", 32, 3)])
def test_values_near_the_largest(rows, cache, d, m):
    """Sums of weights times values stay in range where the values do: one of 2^120 among ordinary ones, a whole row of them, and their negatives."""
    c = Paged(cache, rows, [50, 90], [m, m], kv_heads=2, d=d, seed=11)
    c.fill()
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for at, x in ((3, 2.0 ** 120), (20, -2.0 ** 120), (49, 1.75 * 2.0 ** 119)):
        kr, vr = c.random_rows(1), c.random_rows(1)
        vr[:, :, :d if at == 49 else 1] = x
        c.kv.write(0, c.dev[0][:1].contiguous(), one, torch.tensor([at], dtype=torch.int32, device="cuda"), kr, vr)
    q = c.random_rows(2 * m, 2)
    c.check(c.attend(q, d ** -0.5, m), q, d ** -0.5)


def test_two_caches_on_two_streams_and_in_two_graphs():
    """Each has its own workspace: work that overlaps gives what it gives alone."""
    cs = [Paged("fp8", "bf16", [3000, 500], [m, m], kv_heads=4, group=2, d=128, width=1, seed=m) for m in (4, 40)]
    qs, want, graphs, outs = [], [], [], []
    for c, m in zip(cs, (4, 40)):
        c.fill()
        qs.append(c.random_rows(2 * m, 8))
        want.append(c.attend(qs[-1], 0.09, m))
        outs.append(torch.empty_like(qs[-1]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for c, m, q, out, s in zip(cs, (4, 40), qs, outs, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            for _ in range(5):
                c.attend(q, 0.09, m, out=out)
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o.fill_(-1)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        for c, m, q, s in zip(cs, (4, 40), qs, streams):
            with torch.cuda.stream(s):
                late = [c.attend(q, 0.09, m) for _ in range(5)]
            s.synchronize()
            assert all(torch.equal(x, want[cs.index(c)]) for x in late)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_threads_that_share_a_cache():
    """Rows in and out from several threads, each with a page table of its own."""
    import threading
    c = Paged("bf16", "bf16", [0] * 4, [40] * 4, kv_heads=2, d=64)
    c.fill()
    start, zero = torch.tensor([0, 40], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    tables = [c.dev[0][b:b + 1].contiguous() for b in range(4)]
    want = [c.kv.read(0, t, start, zero, 40) for t in tables]
    torch.cuda.synchronize()
    wrong = []

    def work(b):
        torch.cuda.set_device(0)
        for _ in range(200):
            k, v = c.kv.read(0, tables[b], start, zero, 40)
            c.kv.write(0, tables[b], start, zero, k.to(torch.bfloat16), v.to(torch.bfloat16))
        if not (torch.equal(k, want[b][0]) and torch.equal(v, want[b][1])):
            wrong.append(b)

    threads = [threading.Thread(target=work, args=(b,)) for b in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_refusals_of_the_binding():
    import paper_2312_11462_amd as P
    c = Paged("bf16", "bf16", [3], [2], kv_heads=2, group=2, d=64)
    t, s, cl = c.dev
    q, k = c.random_rows(2, 4), c.random_rows(2)
    c.kv.write(0, t, s, cl, k, k)
    with pytest.raises(ValueError):
        c.kv.attention(0, t.cpu(), s, cl, q, 0.1)
    with pytest.raises(ValueError):
        c.kv.attention(0, t, s[:1], cl, q, 0.1)
    with pytest.raises(TypeError):
        c.kv.attention(0, t.long(), s, cl, q, 0.1)
    with pytest.raises(ValueError):
        c.kv.attention(0, t, s, cl, q.cpu(), 0.1)
    with pytest.raises(TypeError):
        c.kv.attention(0, t, s, cl, q.half(), 0.1)
    with pytest.raises(ValueError):
        c.kv.attention(0, t, s, cl, q.transpose(0, 1), 0.1)
    with pytest.raises(ValueError):
        c.kv.attention(0, t, s, cl, q, 0.1, out=torch.empty(3, 4, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        c.kv.attention(0, t, s, cl, q, 0.1, out=torch.empty(2, 4, 64, device="cuda"))
    with pytest.raises(ValueError):
        c.kv.attention(0, t, s, cl, q, 0.1, parent=torch.zeros(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(P.CsdError) as e:
        c.kv.attention(0, t, s, cl, q[:, :3].contiguous(), 0.1)
    assert e.value.status == -1
    with pytest.raises(P.CsdError) as e:
        c.kv.write(1, t, s, cl, k, k)
    assert e.value.status == -1
    with pytest.raises(P.CsdError):
        c.kv.write(0, t, s, cl, k[:1].expand(2, 2, 64), k)               # one row for all: no distance between rows
    with pytest.raises(TypeError):
        c.kv.write(0, t, s, cl, k, k.float())
    with pytest.raises(ValueError):
        c.kv.write(0, t, s, cl, k, k[:1])
    with pytest.raises(ValueError):
        c.kv.commit(t, cl, torch.zeros(2, 3, dtype=torch.int32, device="cuda"), cl)
    with pytest.raises(ValueError):
        P.PagedKv(c.k, c.v, workspace=torch.zeros(1024, dtype=torch.uint8, device="cuda"))
    # no rows at all: nothing happens
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert c.kv.attention(0, t, none, cl, q[:0], 0.1).shape == (0, 4, 64)
    c.kv.write(0, t, none, cl, k[:0], k[:0])
    assert c.kv.read(0, t, none, cl, 0)[0].shape == (0, 2, 64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,group,others", [(1, 1, 0), (16, 1, 0), (2, 4, 0), (5, 5, 0), (32, 1, 0), (41, 1, 0), (9, 8, 0), (70, 1, 0), (64, 4, MORE), (150, 4, MORE)])
def test_infinite_values_among_the_cached_rows(d, m, group, others):
    """Every row attends them, whatever its weight for each: an infinity of that sign, NaN where both signs meet; in tiles that lie far before the block, and beside it."""
    c = Paged("bf16", "bf16", [500, 90] + [0] * others, [m, m] + [9] * others, kv_heads=2, group=group, d=d, seed=m)
    k, v = c.fill()
    places = c.rng.permutation(490)[:24].tolist() + [497, 499]
    features = c.rng.permutation(d)[:26].tolist()
    for x, (at, f) in enumerate(zip(places, features)):
        v[at, :, f] = math.inf if x % 2 else -math.inf
    v[places[0], :, features[1]] = -math.inf                            # (there is an infinity of the other sign)
    whole = torch.tensor(np.concatenate([[0], np.cumsum([t + n for t, n in zip(c.cached, c.new)])]), dtype=torch.int32, device="cuda")
    c.kv.write(0, c.dev[0], whole, torch.zeros(len(c.cached), dtype=torch.int32, device="cuda"), k, v)
    q = c.random_rows(c.total, 2 * group)
    out = c.attend(q, 0.05, m)
    with np.errstate(invalid="ignore"):
        want = c.check(out, q, 0.05)
    got = out.double().cpu().numpy()
    odd = ~np.isfinite(want)
    assert odd[:m].sum() == m * 2 * group * 26 and np.isnan(want).any()
    assert np.array_equal(got[odd], want[odd], equal_nan=True)


def check_closely(c, out, q, scale, u_p, parent=None, sequences=None):
    """As Paged.check, for the rows of these sequences, with the weights off by u_p of themselves: the bound of the kernels that do not round weights to bf16 (0, all in fp32),
    or keep them in two bf16 planes (2^-15: the second plane is off by 2^-8 of itself, and it is at most 2^-7 of the weight)."""
    start, cached, table = c.start, c.cached, c.table
    some = range(len(cached)) if sequences is None else sequences
    k, v = c.values(c.k, c.ks)[0], c.values(c.v, c.vs)[0]
    dev, qq = out.double().cpu().numpy(), q.double().cpu().numpy()
    live = k[np.isfinite(k).all(-1)]
    worst = 0.0
    for b in some:
        a, z = int(start[b]), int(start[b + 1])
        up = parent[a:z] if parent is not None else None
        args = table[b:b + 1], np.array([0, z - a]), cached[b:b + 1], qq[a:z], scale, up
        want, size = O.attention(k, v, *args), O.attention(k, np.abs(v), *args)
        n = cached[b] + z - a
        dot = abs(scale) * np.sqrt((qq[a:z] ** 2).sum(-1)).max(initial=0) * np.sqrt((live ** 2).sum(-1)).max(initial=0)
        e = (c.d + 4) * 2.0 ** -24 * dot + 2.0 ** -21 + n * 2.0 ** -24
        tol = (2.0 ** -8 if c.rows == "bf16" else 2.0 ** -24) * np.abs(want) + 2 * (u_p + e) * size
        worst = max(worst, (np.abs(dev[a:z] - want) / np.maximum(tol, 1e-300)).max(initial=0))
    assert worst <= 1, f"off by {worst:.2f} times the bound"


CLOSE = [("bf16", "bf16", 64, 2.0 ** -15), ("bf16", "bf16", 128, 2.0 ** -15), ("bf16", "fp8", 64, 2.0 ** -15), ("bf16", "fp8", 128, 2.0 ** -15),
         ("bf16", "bf16", 80, 0.0), ("bf16", "fp32", 64, 0.0), ("fp32", "fp32", 64, 0.0), ("fp32", "fp8", 128, 0.0)]


@pytest.mark.parametrize("rows,cache,d,u_p", CLOSE)
@pytest.mark.parametrize("m,group,tree,others", [(1, 1, False, 0), (1, 8, False, 0), (5, 3, False, 0), (16, 1, False, 0), (5, 4, False, 0), (17, 1, True, 0), (32, 1, False, 0), (33, 1, False, 0),
                                                 (5, 8, False, 0), (41, 1, True, 0), (64, 2, False, 0), (41, 4, True, MORE), (64, 4, False, MORE)])
def test_weights_of_reviews_are_not_rounded_to_bf16(rows, cache, d, u_p, m, group, tree, others):
    """Single tokens, blocks and trees of up to 64 rows: outputs small beside the values that they are sums of, in which a rounded weight shows."""
    c = Paged(cache, rows, [700, 230] + [0] * others, [m, m] + [9] * others, kv_heads=2, group=group, d=d, seed=m)
    c.fill()
    parent = np.concatenate([[-1] + [(i - 1) // 2 for i in range(1, n)] for n in c.new]).astype(np.int32) if tree else None
    q = c.random_rows(c.total, 2 * group, loud=False) * 0.25
    out = c.attend(q, d ** -0.5, m, parent)
    check_closely(c, out, q, d ** -0.5, u_p, parent, [0, 1, len(c.cached) - 1])


@pytest.mark.parametrize("cache,d", [("bf16", 64), ("fp8", 128)])
@pytest.mark.parametrize("group,chunk,others", [(1, 65, 0), (4, 300, 0), (8, 100, 0), (2, 300, MORE)])
def test_a_blocks_weights_do_not_depend_on_its_company(cache, d, group, chunk, others):
    """Blocks and single tokens beside a chunk, whose own weights may be rounded to bf16."""
    c = Paged(cache, "bf16", [300, 700, 40, 500, 64] + [0] * others, [1, 5, 64, chunk, 20] + [9] * others, kv_heads=2, group=group, d=d, seed=chunk)
    c.fill()
    q = c.random_rows(c.total, 2 * group, loud=False) * 0.25
    out = c.attend(q, d ** -0.5, chunk)
    check_closely(c, out, q, d ** -0.5, 2.0 ** -15, None, [0, 1, 2, 4])
    check_closely(c, out, q, d ** -0.5, 2.0 ** -8, None, [3])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,group", [(1, 1), (5, 2), (5, 4), (41, 1), (70, 2)])
@pytest.mark.parametrize("power", [-117, -113, 110])
def test_values_whose_scale_is_near_the_ends(d, m, group, power):
    """e4m3 rows of values around 2^power: the scales reach from 2^-126 to 2^120, and the weights are multiplied by them.  In bf16, subnormal from 2^-126 down in steps
    of 2^-133, a product of weight and scale is off by half a step per plane, times codes of at most 3.5, over a sum of weights of at least 2^-8: 2^-123 per key."""
    c = Paged("fp8", "bf16", [20, 9], [m, m], kv_heads=2, group=group, d=d, seed=m)
    n = 29 + 2 * m
    k, v = (torch.tensor(c.rng.standard_normal((n, 2, d)), dtype=torch.float32).to(torch.bfloat16).cuda() for _ in range(2))
    start = torch.tensor([0, 20 + m, n], dtype=torch.int32, device="cuda")
    c.kv.write(0, c.dev[0], start, torch.zeros(2, dtype=torch.int32, device="cuda"), k, v * 2.0 ** (power - 2))
    q = c.random_rows(2 * m, 2 * group)
    out = c.attend(q, d ** -0.5, m)
    kk, vv = c.values(c.k, c.ks)[0], c.values(c.v, c.vs)[0]
    args = c.table, c.start, c.cached, q.double().cpu().numpy(), d ** -0.5
    want, size = O.attention(kk, vv, *args), O.attention(kk, np.abs(vv), *args)
    u_p = 2.0 ** -15 if m <= 64 else 2.0 ** -8
    tol = 2.0 ** -8 * np.abs(want) + 2 * (u_p + 2.0 ** -15) * size + (20 + m) * 2.0 ** -123      # (scores up to 30: their error is below 2^-15)
    worst = (np.abs(out.double().cpu().numpy() - want) / tol).max()
    assert worst <= 1 and np.median(size) > 2.0 ** (power - 5), f"off by {worst:.2f} times the bound"


@pytest.mark.parametrize("rows,cache,d", SPREAD)
def test_trees_without_a_word_on_their_size(rows, cache, d):
    """A batch of more than 64 rows whose trees are within 64 each; a single tree of more is refused."""
    import paper_2312_11462_amd as P
    rng = np.random.default_rng(1)
    c = Paged(cache, rows, [70, 0, 33], [41, 9, 64], kv_heads=2, d=d, seed=3)
    c.fill()
    parent = np.concatenate([[int(rng.integers(max(0, i - 9), i)) if i else -1 for i in range(m)] for m in c.new]).astype(np.int32)
    q = c.random_rows(c.total, 2)
    c.check(c.attend(q, d ** -0.5, None, parent), q, d ** -0.5, parent)
    one = Paged(cache, rows, [5], [65], kv_heads=2, d=d, seed=3)
    one.fill()
    with pytest.raises(P.CsdError) as e:
        one.attend(one.random_rows(65, 2), 0.1, None, np.zeros(65, dtype=np.int32))
    assert e.value.status == -2


@pytest.mark.parametrize("cache,m", [("fp8", 4), ("bf16", 40)])
def test_one_cache_on_two_streams_and_in_two_graphs(cache, m):
    """Sequences that several workgroups share: calls that overlap, eager and replayed, on two streams, give what one alone gives; so do later ones."""
    c = Paged(cache, "bf16", [3000, 500], [m, m], kv_heads=4, group=2, d=128, seed=m)
    c.fill()
    q = [c.random_rows(2 * m, 8) for _ in range(2)]
    want = [c.attend(x, 0.09, m) for x in q]
    outs = [torch.empty_like(x) for x in q]
    torch.cuda.synchronize()
    graphs = []
    for x, out in zip(q, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for _ in range(8):
                c.attend(x, 0.09, m, out=out)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for out in outs:
            out.fill_(-1)
        torch.cuda.synchronize()
        late = [[], []]
        for _ in range(8):
            for i, s in enumerate(streams):
                with torch.cuda.stream(s):
                    late[i].append(c.attend(q[i], 0.09, m))
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], want[i]) and all(torch.equal(x, want[i]) for x in late[i])
            assert torch.equal(c.attend(q[i], 0.09, m), want[i])


def test_threads_that_attend_one_cache():
    """Each on a stream of its own, or all on one."""
    import threading
    m = 4
    c = Paged("bf16", "bf16", [3000, 500], [m, m], kv_heads=4, group=2, d=128, seed=m)
    c.fill()
    q = [c.random_rows(2 * m, 8) for _ in range(4)]
    want = [c.attend(x, 0.09, m) for x in q]
    torch.cuda.synchronize()
    wrong = []

    def work(i, stream):
        torch.cuda.set_device(0)
        with torch.cuda.stream(stream):
            for _ in range(50):
                if not torch.equal(c.attend(q[i], 0.09, m), want[i]):
                    wrong.append(i)

    one = torch.cuda.Stream()
    for streams in ([torch.cuda.Stream() for _ in range(4)], [one] * 4):
        threads = [threading.Thread(target=work, args=(i, s)) for i, s in enumerate(streams)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not wrong


def test_a_workspace_that_is_given_is_the_one_that_is_used():
    import paper_2312_11462_amd as P
    from paper_2312_11462_amd.binding import PAGED_WORKSPACE_BYTES
    c = Paged("bf16", "bf16", [3000], [4], kv_heads=4, d=64, seed=1)
    c.fill()
    q = c.random_rows(4, 4)
    want = c.attend(q, 0.1, 4)
    w = torch.zeros(PAGED_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    kv = P.PagedKv(c.k, c.v, workspace=w)
    assert torch.equal(kv.attention(0, *c.dev, q, 0.1, 4), want) and w.any()      # (parts of the split sequence lie there)


@pytest.mark.parametrize("rows,cache,d,made", [("fp32", "fp32", 64, 0), ("fp32", "fp8", 64, 0), ("bf16", "bf16", 80, 0), ("bf16", "fp32", 64, 0), ("bf16", "bf16", 64, 1), ("bf16", "fp8", 128, 1)])
def test_a_cache_has_a_workspace_only_where_its_attention_uses_one(rows, cache, d, made):
    from paper_2312_11462_amd.binding import PAGED_WORKSPACE_BYTES
    c = Paged(cache, rows, [40], [3], kv_heads=2, d=d)
    c.fill()
    q = c.random_rows(3, 2)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    out = c.attend(q, 0.1, 3)
    del out
    assert (torch.cuda.memory_allocated() - before) // PAGED_WORKSPACE_BYTES == made


@pytest.mark.parametrize("rows,cache,d", [("fp32", "fp32", 32), ("bf16", "bf16", 80), ("bf16", "bf16", 64), ("bf16", "bf16", 128)])
@pytest.mark.parametrize("m", [2, 40, 70])
def test_rows_whose_scores_are_all_minus_infinity(rows, cache, d, m):
    """0 / 0, as the formula has it, however many pages are gone; a row without any key left is zero, without a search for one."""
    c = Paged(cache, rows, [300, 300, 300], [m, m, m], kv_heads=2, d=d, seed=m)
    k, v = c.fill()
    k[:300 + m, 1, 3] = -math.inf                                       # the first sequence's second head
    whole = torch.arange(4, dtype=torch.int32, device="cuda") * (300 + m)
    c.kv.write(0, c.dev[0], whole, torch.zeros(3, dtype=torch.int32, device="cuda"), k, v)
    c.table[0, 3:15] = -1
    c.table[1] = -1
    c.dev[0].copy_(torch.tensor(c.table))
    q = c.random_rows(3 * m, 2).abs()
    out = c.attend(q, d ** -0.5, m)
    with np.errstate(invalid="ignore"):
        want = c.check(out, q, d ** -0.5)
    assert np.isnan(want[:m, 1]).all() and torch.isnan(out[:m, 1]).all() and (out[m:2 * m] == 0).all() and torch.isfinite(out[2 * m:]).all()


EVERY = FULL + [("fp32", "fp32", 64), ("fp32", "fp8", 64), ("bf16", "bf16", 80)]


@pytest.mark.parametrize("rows,cache,d", EVERY)
@pytest.mark.parametrize("m,group,others", [(1, 1, 0), (1, 8, 0), (5, 4, 0), (9, 2, 0), (40, 1, 0), (64, 2, 0), (130, 1, 0), (40, 4, MORE), (150, 4, MORE)])
def test_every_key_counts_once(rows, cache, d, m, group, others):
    """All weights alike, and of each stretch of 32 keys a feature that is 1 while the others are 0 (the first head counts the stretches by d, the second their rounds): an output
    is the share of its stretches' keys.  Weights and their sums are exact then, and a key left out at a border of tiles, pages, shares or parts, or taken twice, changes
    its share by more than the output's rounding (one of 141 keys at least) or is in a share that has to be 0."""
    lens = [9001, 3, 4097, 0, 1333]
    c = Paged(cache, rows, lens + [0] * others, [m] * 5 + [9] * others, kv_heads=2, group=group, d=d, page=16 if m % 2 else 64, seed=m)
    k, _ = c.fill()
    whole = [t + n for t, n in zip(c.cached, c.new)]
    stretch = np.concatenate([np.arange(n) for n in whole]) // 32
    feature = np.stack([stretch % d, stretch // d % d], 1)
    v = torch.nn.functional.one_hot(torch.tensor(feature), d).to(TORCH[rows]).cuda()
    start = torch.tensor(np.concatenate([[0], np.cumsum(whole)]), dtype=torch.int32, device="cuda")
    c.kv.write(0, c.dev[0], start, torch.zeros(len(whole), dtype=torch.int32, device="cuda"), k, v)
    lost = range(20, 23)
    c.table[4, lost] = -1
    c.dev[0].copy_(torch.tensor(c.table))
    q = c.random_rows(c.total, 2 * group)
    got = c.attend(q, 0.0, m).double().cpu().numpy()
    for b, t in enumerate(lens):
        there = np.ones(t + m)
        if b == 4:
            there[20 * c.page:23 * c.page] = 0
        at = np.arange(t + m) // 32
        for head, f in enumerate((at % d, at // d % d)):
            counts = np.zeros((t + m, d))
            counts[np.arange(t + m), f] = there
            want = np.cumsum(counts, 0)[t:] / np.cumsum(there)[t:, None]
            off = np.abs(got[c.start[b]:c.start[b + 1], head * group:(head + 1) * group] - want[:, None])
            assert (off <= (2.0 ** -8 if rows == "bf16" else 2.0 ** -24) * 1.001 * want[:, None] + 2.0 ** -22 * want[:, None]).all(), (b, head)


@pytest.mark.parametrize("rows,cache,d", EVERY)
@pytest.mark.parametrize("m,group,others", [(1, 2, 0), (5, 4, 0), (64, 1, 0), (129, 1, 0), (200, 2, MORE)])
def test_errors_are_those_of_the_roundings(rows, cache, d, m, group, others):
    """Over all outputs.  Roundings to bf16 are off by 2^-8 / sqrt(3) of the step's lower end at most in the mean square, independently of one another: the output's, of itself, and in chunks of
    more than 64 rows each weight's, of p v.  With the mean over the step's mantissas (1 / m^2 over m in 1 .. 2, density 1 / (m ln 2): 0.54) that is 0.42 of 2^-8; held to 0.55."""
    c = Paged(cache, rows, [9001, 1200] + [0] * others, [m] * 2 + [9] * others, kv_heads=2, group=group, d=d, seed=m)
    c.fill()
    q = c.random_rows(c.total, 2 * group, loud=False)
    got = c.attend(q, d ** -0.5, m).double().cpu()
    kk, vv = (torch.tensor(c.values(pool, scale)[0]) for pool, scale in ((c.k, c.ks), (c.v, c.vs)))
    rounded = 2.0 ** -8 if rows == "bf16" else 0.0
    weights = rounded if m > 64 and d in (64, 128) and rows == "bf16" else 2.0 ** -14 if rows == "bf16" else 2.0 ** -16
    err = room = 0.0
    for b in range(2):
        n = c.cached[b] + m
        page, slot = torch.tensor(c.table[b])[torch.arange(n) // c.page].long(), torch.arange(n) % c.page
        hidden = torch.arange(n)[None] > c.cached[b] + torch.arange(m)[:, None]
        for h in range(2 * group):
            k, v = kk[page, h // group, slot], vv[page, h // group, slot]
            p = ((q[c.start[b]:c.start[b + 1], h].double().cpu() @ k.t().contiguous()) * d ** -0.5).masked_fill(hidden, -math.inf).softmax(-1)
            want = p @ v
            err += ((got[c.start[b]:c.start[b + 1], h] - want) ** 2).sum().item()
            room += (0.55 ** 2 * (rounded ** 2 * want ** 2 + weights ** 2 * (p ** 2 @ v ** 2))).sum().item()
    assert err <= room, f"{math.sqrt(err / room):.2f} times the bound"


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("rows", ["fp32", "bf16"])
def test_attention_over_a_models_rows_is_the_models_own(rows, tree):
    """Its first layer computed in 64 bits around the attention over pages that hold its cached rows, against what the model itself computed.  With fp32 queries both attentions
    are exact but for 2^-15 or so (the model's products take two bf16 planes); bf16 queries and outputs are off by 2^-9 in the mean."""
    import csd_inputs as I
    import paper_2312_11462_amd as P
    H, dh, n, m = 4, 64, 96, 7
    shape = I.ModelShape("own", 0, "bf16", 1, 256, H, dh, 512, 1024)
    weights = I.make_weights(shape, 5, device="cuda", std=0.08)
    gm = P.Model(shape, weights, max_batch=1, max_seq=160, max_block=8)
    toks = I.token_ids(120, shape.vocab, 5, 1).cuda()
    for pos in range(0, n, 8):
        gm.verify_block(toks[None, pos:pos + 8].contiguous(), torch.full((1,), pos, dtype=torch.int32, device="cuda"))
    trace = torch.zeros((2, m, 256), device="cuda")
    block, at = toks[None, n:n + m].contiguous(), torch.full((1,), n, dtype=torch.int32, device="cuda")
    parent = torch.tensor([0, 0, 0, 1, 1, 2, 4], dtype=torch.int32, device="cuda")
    depth = torch.tensor([0, 1, 1, 2, 2, 2, 3] if tree else range(m))
    gm.set_trace(trace)
    if tree:
        gm.verify_tree(block, parent[None].contiguous(), at)
    else:
        gm.verify_block(block, at)
    gm.set_trace(None)
    pool = torch.zeros((1, 8, H, 16, dh), dtype=torch.bfloat16, device="cuda")
    kv = P.PagedKv(pool, torch.zeros_like(pool))
    table = torch.tensor([[5, 0, 7, 2, 1, 6, 3]], dtype=torch.int32, device="cuda")
    K, V = gm.kv_read(0, 0, 0, n + m)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv.write(0, table, torch.tensor([0, n + m], dtype=torch.int32, device="cuda"), zero, K.view(n + m, H, dh), V.view(n + m, H, dh))
    embed, norm, wq, _, _, wo, norm2, gate, up, down = (w.double().cpu() for w in weights[:10])

    def rms(x, g):
        return x / (x.square().mean(-1, keepdim=True) + shape.rms_eps).sqrt() * g

    x = embed[block[0].long().cpu()]
    q = (rms(x, norm) @ wq).view(m, H, dh)
    angle = (n + depth.double())[:, None] * shape.rope_theta ** (-2 * torch.arange(dh // 2, dtype=torch.float64) / dh)
    a, b = q.chunk(2, -1)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    q = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    out = kv.attention(0, table, torch.tensor([0, m], dtype=torch.int32, device="cuda"), at, q.to(TORCH[rows]).cuda(), dh ** -0.5, m, parent=parent if tree else None)
    x = x + out.double().cpu().reshape(m, H * dh) @ wo
    h = rms(x, norm2)
    x = x + (torch.nn.functional.silu(h @ gate) * (h @ up)) @ down
    far = ((trace[1].double().cpu() - x).norm() / (x - trace[0].double().cpu()).norm()).item()
    assert far < (2.0 ** -12 if rows == "fp32" else 2.0 ** -7), far
