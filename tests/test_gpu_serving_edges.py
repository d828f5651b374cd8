"""The calls of a serving step where they could go wrong: chunks over tables that their lengths pass, sequences cut inside pages that others use, thousands of
sequences, rows of equal logits, borders among tokens of equal weight.  The plain forms are oracle/serving.py's; the bounds are test_gpu_serving's."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import serving as O
from test_gpu_paged import Paged
from test_gpu_serving import Both, States, as_sets, logits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2312_11462_amd as P
    P.lib()


# ------------------------------------------------------------------------------------------------ chunks over tables that their lengths pass

def over_the_table(cls, cache, d, entries, what):
    """A chunk of 260 rows, 64 x 8 heads (so many items that whole workgroups of rows take them), of a sequence whose table ends behind so many pages of 16 rows."""
    c = cls(cache, "bf16", [16 * entries], [260], kv_heads=64, group=8, d=d, seed=entries) if cls is States else \
        cls(cache, "bf16", [16 * entries], [0], kv_heads=64, group=8, d=d, seed=entries)
    if cls is Paged:
        c.fill()
        c.dev[1] = torch.tensor([0, 260], dtype=torch.int32, device="cuda")
    assert c.table.shape[1] == entries
    last = int(c.table[0, entries - 1])
    c.v[0, last, 0, 15, 3] = what                            # the last position of all; every row attends it
    c.v[0, last, 1, 7, d - 1] = -what
    return c


@pytest.mark.parametrize("cls", [States, Paged], ids=["cross", "self"])
@pytest.mark.parametrize("entries,length", [(1, 64), (3, 64), (3, 1 << 20), (3, 2 ** 31 - 300), (5, 127), (5, 128), (5, 4096), (4, 64), (4, 200)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", [1.0, math.inf])
def test_chunks_of_sequences_longer_than_their_tables(cls, entries, length, d, what):
    """What lies behind the table's last row is no row, however long the sequence is said to be: the rows attend what the table names, once each."""
    c = over_the_table(cls, "bf16", d, entries, what)
    c.dev[2] = torch.tensor([length], dtype=torch.int32, device="cuda")
    q = c.random_rows(260, heads=512)
    out = (c.cross(q, d ** -0.5, 260) if cls is States else c.attend(q, d ** -0.5, 260))[:, :16].double().cpu()
    for kv in range(2):
        k, v = (torch.tensor(x[0][c.table[0], kv].reshape(16 * entries, d)) for x in (c.values(c.k, c.ks), c.values(c.v, c.vs)))
        qq = q[:, 8 * kv:8 * kv + 8].double().cpu().reshape(-1, d)
        p = torch.softmax(qq @ k.t().contiguous() * d ** -0.5, -1)
        want, size, got = p @ v, p @ v.abs(), out[:, 8 * kv:8 * kv + 8].reshape(-1, d)
        fine = torch.isfinite(want)
        assert torch.equal(got[~fine], want[~fine]) and int((~fine).sum()) == (260 * 8 if math.isinf(what) else 0)
        e = (d + 4) * 2.0 ** -24 * float(qq.norm(dim=-1).max() * k.norm(dim=-1).max()) * d ** -0.5 + 2.0 ** -21 + 16 * entries * 2.0 ** -24
        assert ((got - want).abs()[fine] <= (2.0 ** -8 * want.abs() + 2 * (2.0 ** -8 + e) * size)[fine]).all()


# ------------------------------------------------------------------------------------------------ weights of chunks

@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,kv_heads,group", [(1, 2, 1), (64, 2, 2), (65, 2, 1), (100, 2, 8), (300, 2, 2), (260, 64, 8), (700, 80, 1)])
def test_weights_over_an_encoder_are_not_rounded_to_bf16(m, kv_heads, group, d, cache):
    """Tokens, blocks and chunks in every kernel: outputs small beside the values that they are sums of, in which a rounded weight shows."""
    c = States(cache, "bf16", [700, 230], [m, m], kv_heads=kv_heads, group=group, d=d, seed=m + d)
    q = c.random_rows(c.total, heads=kv_heads * group, loud=False) * 0.25
    out = c.cross(q, d ** -0.5, m)
    kk, vv = (torch.tensor(c.values(pool, scale)[0]) for pool, scale in ((c.k, c.ks), (c.v, c.vs)))
    for b, n in enumerate(c.cached):
        page, slot = torch.tensor(c.table[b])[torch.arange(n) // c.page].long(), torch.arange(n) % c.page
        for h in range(2 * group):
            qq, got = (x[c.start[b]:c.start[b + 1], h].double().cpu() for x in (q, out))
            k, v = kk[page, h // group, slot], vv[page, h // group, slot]
            p = torch.softmax(qq @ k.t().contiguous() * d ** -0.5, -1)
            e = (d + 4) * 2.0 ** -24 * float(qq.norm(dim=-1).max() * k.norm(dim=-1).max()) * d ** -0.5 + 2.0 ** -21 + n * 2.0 ** -24
            tol = 2.0 ** -8 * (p @ v).abs() + 2 * (2.0 ** -15 + e) * (p @ v.abs())
            off = ((got - p @ v).abs() / tol).max().item()
            assert off <= 1, f"off by {off:.2f} times the bound"


# ------------------------------------------------------------------------------------------------ pages that others use

def test_rows_of_shared_pages_are_nobodys_to_write():
    """The one that took the pages, then the one that gave them, is cut inside a shared page: neither gets rows there; back at the page's first row it does."""
    c = Both(12, 16, 3, 5, seed=1)
    c.plan([0, 0, 0], [48, 0, 0], 48)
    c.share([-1, 0, -1], [0, 48, 0])
    c.release([-1, 40, -1])
    shared = set(c.ref.table[0][:3])
    want = c.plan([48, 40, 0], [1, 8, 2], 16)
    assert want[4] == [1, 0, 1] and want[0] == [0, 1, 1, 3]
    assert not {s // 16 for s in want[3] if s >= 0} & shared
    assert c.plan([48, 40, 0], [0, 0, 0], 4)[4] == [1, 1, 1]
    c.release([40, -1, 0])
    assert c.plan([40, 40, 0], [3, 3, 3], 16)[4] == [0, 0, 1]
    c.release([-1, 32, 0])
    assert c.plan([40, 32, 0], [3, 16, 0], 19)[4] == [1, 1, 1]
    assert c.plan([10, 8, 0], [30, 70, 0], 130)[4] == [0, 0, 1]
    c.release([-1, 0, -1])
    assert c.plan([10, 0, 0], [30, 0, 0], 30)[4] == [1, 1, 1]


@pytest.mark.parametrize("entries,at", [(9, 8), (9, 3), (40, 38), (40, 1)])
def test_a_shared_page_anywhere_among_the_rows_to_be_written(entries, at):
    """A caller that has shared one page of a sequence by itself; the rows begin before it, in it, behind it and end before it."""
    c = Both(2 * entries, 16, 2, entries, seed=entries + at)
    c.plan([0, 0], [16 * entries, 0], 16 * entries)
    c.ref.users[c.ref.table[0][at]] += 1
    c.gpu.users[c.ref.table[0][at]] += 1
    for t, n, served in ((0, 16 * entries, 0), (16 * at + 15, 1, 0), (16 * at - 1, 2, 0), (16 * at - 1, 1, 1), (0, 16 * at, 1), (16 * at + 16, 16 * (entries - at - 1), 1)):
        assert c.plan([t, 0], [n, 0], 16 * entries)[4][0] == served, (t, n)


@pytest.mark.parametrize("sequences,page", [(40, 16), (300, 32), (1500, 16), (2100, 64)])
def test_shared_prompts_that_are_cut_anywhere(sequences, page):
    """Every third sequence has a prompt that others take over; all are cut at any length, go back to a page's first row where they get no rows, and end."""
    c = Both(sequences * 8, page, sequences, 8, seed=sequences)
    rng, b = c.rng, np.arange(sequences)
    giver = b % 3 == 0
    length = np.where(giver, rng.integers(1, 5 * page, sequences), 0)
    c.plan(np.zeros(sequences, dtype=int), length, int(length.sum()))
    source = np.where(giver, -1, b - b % 3)
    c.share(source, length[source])
    length = np.where(giver, length, np.array(c.ref.held) * page)
    for step in range(4):
        cut = np.where(rng.random(sequences) < 0.4, (length * rng.random(sequences)).astype(int), length)
        c.release(np.where(cut < length, cut, -1))
        length = cut
        new = rng.integers(0, 3 * page // 2, sequences)
        served = np.array(c.plan(length, new, int(new.sum()))[4])
        assert 0 < served.sum() < sequences or step
        length = length + new * served
        stuck = (served == 0) & (rng.random(sequences) < 0.7)
        length = np.where(stuck, length // page * page, length)
        c.release(np.where(stuck, length, -1))
        used = {}
        for s, row in enumerate(c.ref.table):
            for x in row[:c.ref.held[s]]:
                used[x] = used.get(x, 0) + 1
        assert all(c.ref.users[x] == n for x, n in used.items())
    c.release(np.zeros(sequences, dtype=int))
    assert int(c.gpu.n_free) == c.ref.n_pages and not c.gpu.users.any()


def test_thousands_of_sequences_most_of_them_without_rows():
    """More sequences than the row kernel keeps the starts of in LDS; runs of sequences without rows, at both ends too, and rows behind the last."""
    for sequences, share in ((4096, 0.5), (4097, 0.5), (5000, 0.02), (9001, 0.6)):
        c = Both(3 * sequences, 16, sequences, 4, seed=sequences)
        new = np.where(c.rng.random(sequences) < share, c.rng.integers(1, 40, sequences), 0)
        new[:17] = new[-70:] = 0
        length = c.rng.integers(0, 25, sequences)
        rows = int(new.sum())
        assert sum(c.plan(length, new, rows + 300)[4]) == sequences
        c.plan(length + new, np.ones(sequences, dtype=int), sequences)
        c.release(np.where(c.rng.random(sequences) < 0.3, -1, length))
        c.release(np.zeros(sequences, dtype=int))
        assert int(c.gpu.n_free) == c.ref.n_pages


# ------------------------------------------------------------------------------------------------ sets and draws at their borders

def strictly(x, u=None, **kw):
    """Draws and filters rows x and looks at every token: one that stays where the plain form leaves it out, or the other way round, has to lie at a border within
    the sums' error E (or weigh nothing); the probabilities and the draw go by the set that the kernel kept."""
    import paper_2312_11462_amd as P
    rows, V = x.shape
    if u is None:
        u = torch.tensor(np.random.default_rng(V).integers(0, 1 << 24, rows) * 2.0 ** -24, dtype=torch.float32).cuda()
    probs = torch.full((rows, V), -1.0, device="cuda")
    tokens = P.sample(x, u, probs=probs, **kw).tolist()
    assert torch.equal(probs, P.filter_probs(x, **kw)) and P.sample(x, u, **kw).tolist() == tokens
    p, xx, uu = probs.cpu().numpy().astype(np.float64), x.double().cpu().numpy(), u.cpu().numpy()
    sets = as_sets(rows, *(kw.get(n, d) for n, d in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))))
    E, largest = 2 * V * 2.0 ** -45, torch.finfo(x.dtype).max
    for r in range(rows):
        (w, slack), (full, _) = O.weights(xx[r], *sets[r], largest=largest), O.weights(xx[r], sets[r][0], largest=largest)
        kept, name = p[r] > 0, f"row {r} {sets[r]}"
        if not full.sum() > 0:
            assert tokens[r] == -1 and not p[r].any(), name
            continue
        other = np.flatnonzero((kept != (w > 0)) & ~(slack <= E) & ~(~kept & (w <= 2.0 ** -45)))
        assert not len(other), f"{name}: tokens {other[:8]} stay or go"
        full = np.where(kept, full, 0.0)
        z = full.sum()
        tol = full / z * (2.0 ** -24 + 2 * E / z) + 2.0 ** -45
        assert (np.abs(p[r] - full / z) <= tol).all(), f"{name}: off by {(np.abs(p[r] - full / z) / tol).max():.2f} times the bound"
        at, run, t = min(max(float(uu[r]), 0.0), 1 - 2.0 ** -24) * z, np.cumsum(full), tokens[r]
        assert 0 <= t < V and kept[t] and run[t] - full[t] <= at + E and at - E < run[t], f"{name}: token {t} for u {uu[r]}"


LIMITS = [dict(), dict(temperature=0.0), dict(top_k=40), dict(top_k=193), dict(top_p=0.9), dict(top_p=0.5), dict(min_p=0.05), dict(top_k=50, top_p=0.8),
          dict(temperature=1.7, top_k=300, top_p=0.95, min_p=0.01), dict(top_k=900, top_p=0.37), dict(top_p=0.5, min_p=0.5)]


@pytest.mark.parametrize("kw", LIMITS, ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_token_that_stays_or_goes(dtype, kw):
    for V in (1, 5, 255, 1000, 4099, 32000):
        strictly(logits(4, V, dtype, V + 3, likely=min(V, 20)), **kw)
    strictly(logits(2, 131072, dtype, 8), **kw)


@pytest.mark.parametrize("kw", LIMITS, ids=str)
@pytest.mark.parametrize("V,levels", [(1000, 1), (1000, 2), (32000, 1), (32000, 3), (32000, 40), (5000, 700)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_token_that_stays_or_goes_among_equal_ones(V, levels, dtype, kw):
    x = torch.randint(0, levels, (3, V), generator=torch.Generator().manual_seed(V + levels)).float() * 0.125 - 2.0
    x[2, ::5] = -math.inf
    strictly(x.to(dtype).cuda(), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_token_that_stays_or_goes_by_settings_of_its_own(dtype):
    g = torch.Generator().manual_seed(5)
    for rows, V in ((300, 700), (24, 32000)):
        k = torch.randint(-3, 400, (rows,), generator=g, dtype=torch.int32)
        t, p, m = torch.rand(rows, generator=g) * 1.5, torch.rand(rows, generator=g) * 1.2, torch.rand(rows, generator=g) * 0.3 - 0.1
        t[::7] = 0
        strictly(logits(rows, V, dtype, 17), temperature=t.cuda(), top_k=k.cuda(), top_p=p.cuda(), min_p=m.cuda())


@pytest.mark.parametrize("V", [1, 7, 1000, 1024, 32000, 131072, 1 << 18])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sets_and_draws_of_equal_logits_are_exact(V, dtype):
    """All weights are 1, so every sum is a whole number: the first k tokens, the first ceil(p k) of those, and token floor(u n) of n.  (2^18 weights make 2^63.)"""
    import paper_2312_11462_amd as P
    half = [i / 512 for i in range(0, 512, 37)]
    u = [0.0, 2.0 ** -24, 0.25, 0.5, 0.5 - 2.0 ** -24, 1 - 2.0 ** -24] + half
    x = torch.full((len(u), V), 0.75, dtype=dtype, device="cuda")
    for k, p in ((0, 1.0), (0, 0.5), (0, 0.37), (0, 1 - 2.0 ** -24), (7, 1.0), (300, 1.0), (900, 0.37), (193, 0.5), (0, 0.0), (1024, 0.5)):
        first = min(k, V) if k > 0 else V
        n = max(math.ceil(Fraction(float(np.float32(p))) * first), 1)
        tokens, probs = (f(x, *a, top_k=k, top_p=p) for f, a in ((P.sample, (torch.tensor(u, dtype=torch.float32, device="cuda"),)), (P.filter_probs, ())))
        assert tokens.tolist() == [math.floor(Fraction(a) * n) for a in u], (k, p)
        assert (probs[:, :n] == np.float32(1 / n)).all() and not probs[:, n:].any(), (k, p)


@pytest.mark.parametrize("V", [131072, 131069])
@pytest.mark.parametrize("rows,dtype", [(160, torch.float32), (210, torch.bfloat16)])
def test_rows_of_large_batches_are_those_of_small_ones(rows, dtype, V):
    """So many probabilities that they are stored past the caches: the same bits, and nothing beside them."""
    import paper_2312_11462_amd as P
    x = logits(rows, V, dtype, 31)
    x[rows // 2] = -math.inf
    for kw in (dict(), dict(temperature=0.0), dict(top_k=50, top_p=0.9), dict(top_p=0.9), dict(top_p=0.2), dict(min_p=0.05), dict(top_k=5000)):
        out = torch.full((rows * V + 64,), 7.0, device="cuda")
        probs = P.filter_probs(x, out=out[32:-32].view(rows, V), **kw)
        assert (out[:32] == 7).all() and (out[-32:] == 7).all()
        for at in range(0, rows, 70):
            assert torch.equal(probs[at:at + 70], P.filter_probs(x[at:at + 70], **kw)), (kw, at)


def test_numbers_that_the_parameters_types_do_not_hold():
    import paper_2312_11462_amd as P
    x, u = logits(3, 700, torch.float32, 2), torch.tensor([0.1, 0.5, 0.9], device="cuda")
    for k in (2 ** 31, 2 ** 40, 2 ** 63 - 1, -2 ** 40):
        assert torch.equal(P.filter_probs(x, top_k=k, top_p=0.9), P.filter_probs(x, top_p=0.9)) and torch.equal(P.sample(x, u, top_k=k), P.sample(x, u))
    assert torch.equal(P.filter_probs(x, temperature=1e39), P.filter_probs(x, temperature=math.inf))       # (logits of a few units: all alike)
    assert torch.equal(P.filter_probs(x, top_p=1e300), P.filter_probs(x))
    for bad in (dict(top_k=5.5), dict(temperature="warm"), dict(top_p=[0.9])):
        with pytest.raises(TypeError):
            P.sample(x, u, **bad)
    for bad in (dict(temperature=-1e39), dict(top_p=-1e39), dict(min_p=1e39), dict(temperature=math.nan, top_k=2 ** 40)):
        with pytest.raises(P.CsdError):
            P.sample(x, u, **bad)
