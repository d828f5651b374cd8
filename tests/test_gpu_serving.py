"""Draws from logits, page plans and cross-attention over pages on the GPU against the plain forms in 64 bits (oracle/serving.py).

Bounds.  A weight is a whole number of 2^-45: off by at most 2^-46, and by the error of its exponential, 2^-47 of it and 46 * 2^-52 from its argument: by less than
2^-45 in all.  So a sum of weights over V tokens is off by at most V * 2^-45, and what two sums decide may only differ where they are nearer than
E = 2 V * 2^-45.  A probability w / sum is rounded once to fp32 (2^-24 of it).
"""
import math

import numpy as np
import pytest
import torch

from oracle import serving as O
from test_gpu_paged import Paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2312_11462_amd as P
    P.lib()


# ------------------------------------------------------------------------------------------------ draws

def check_rows(x, tokens, probs, u, sets, dtype=torch.float32):
    """x [rows][V] float64 as the kernel read them; sets: (temperature, top_k, top_p, min_p) of every row."""
    V = x.shape[1]
    E = 2 * V * 2.0 ** -45
    for r in range(len(x)):
        w, slack = O.weights(x[r], *sets[r], largest=torch.finfo(dtype).max)
        if probs is not None:
            p = probs[r].astype(np.float64)
            assert (p >= 0).all(), r
            other = (p > 0) != (w > 0)
            assert (slack[other] <= E).all() or (w[other & (slack > E)] <= 2.0 ** -45).all(), f"row {r} {sets[r]}: tokens {np.flatnonzero(other)[:8]} stay or go"
            if w.sum() > 0 and not (slack[other] <= E).any():
                want = w / w.sum()
                tol = want * (2.0 ** -24 + 2 * E / w.sum()) + 2.0 ** -45
                assert (np.abs(p - want) <= tol).all(), f"row {r} {sets[r]}: off by {(np.abs(p - want) / tol).max():.2f} times the bound"
        if tokens is not None:
            if not w.sum() > 0:
                assert tokens[r] == -1, r
                continue
            if (slack <= E).any():
                continue                                    # (a border that rounding may move)
            t, z = int(tokens[r]), w.sum()
            assert 0 <= t < V and w[t] > 0, f"row {r} {sets[r]}: token {t} has no weight"
            at = min(max(float(u[r]), 0.0), 1 - 2.0 ** -24) * z
            run = np.cumsum(w)
            assert run[t] - w[t] <= at + E and at - E < run[t], f"row {r} {sets[r]}: token {t} for u {u[r]}"


def as_sets(rows, temperature, top_k, top_p, min_p):
    def of(v, r):
        return v if not isinstance(v, torch.Tensor) else v.flatten()[r * v.numel() // rows].item()
    f32 = np.float32
    return [(float(f32(of(temperature, r))), int(of(top_k, r)), float(f32(of(top_p, r))), float(f32(of(min_p, r)))) for r in range(rows)]


def run_rows(x, u=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, expect_same=True):
    """Draws and filters rows x [rows][V], checks both against the oracle and against one another; returns (tokens, probs)."""
    import paper_2312_11462_amd as P
    rows, V = x.shape
    if u is None:
        u = torch.tensor(np.random.default_rng(rows * V).integers(0, 1 << 24, rows) * 2.0 ** -24, dtype=torch.float32).cuda()
    kw = dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    tokens, probs = P.sample(x, u, **kw), P.filter_probs(x, **kw)
    both = torch.full((rows, V), -1.0, device="cuda")
    again = P.sample(x, u, probs=both, **kw)
    assert torch.equal(again, tokens) and torch.equal(both, probs)
    check_rows(x.double().cpu().numpy(), tokens.cpu().numpy(), probs.cpu().numpy(), u.cpu().numpy(), as_sets(rows, temperature, top_k, top_p, min_p), x.dtype)
    return tokens, probs


def logits(rows, V, dtype, seed=0, spread=2.0, likely=20):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn(rows, V, generator=g)
    at = torch.randint(0, V, (rows, likely), generator=g)
    x.scatter_(1, at, 6.0 + 2.0 * torch.randn(rows, likely, generator=g))
    return x.to(dtype).cuda()


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.6), dict(top_k=1), dict(top_k=40), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=50, top_p=0.8),
            dict(temperature=1.7, top_k=300, top_p=0.95, min_p=0.01), dict(temperature=0.3, top_p=0.999), dict(top_p=0.0), dict(min_p=1.0), dict(top_k=1 << 30, top_p=1.0)]


@pytest.mark.parametrize("kw", SETTINGS, ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 255, 512, 1000, 4099])
def test_small_vocabularies(V, dtype, kw):
    run_rows(logits(5, V, dtype, V), **kw)


@pytest.mark.parametrize("rows", [3, 600])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_vocabularies_of_a_few_pieces(rows, dtype):
    for V in (4, 5, 6, 7, 8, 9, 10, 13, 15, 16, 17, 31, 255, 256, 257, 511, 513, 1023, 1025, 4096, 4097, 8191, 8193):
        for kw in (dict(), dict(top_k=5, top_p=0.9)):
            run_rows(logits(rows, V, dtype, V, likely=4)[:3 if V > 600 else rows], **kw)


@pytest.mark.parametrize("kw", [SETTINGS[i] for i in (0, 1, 4, 5, 8)], ids=str)
@pytest.mark.parametrize("V,dtype", [(32000, torch.float32), (32128, torch.bfloat16), (50001, torch.float32), (65537, torch.bfloat16), (131072, torch.float32),
                                     (131072, torch.bfloat16), (1 << 18, torch.float32), (1 << 18, torch.bfloat16)])
def test_large_vocabularies(V, dtype, kw):
    run_rows(logits(3, V, dtype, V + 1), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V", [(300, 700), (600, 2003), (300, 9001), (40, 32000)])
def test_every_row_has_its_own_settings(rows, V, dtype):
    g = torch.Generator().manual_seed(rows)
    t = torch.rand(rows, generator=g) * 1.5
    t[::7] = 0
    k = torch.randint(-3, 200, (rows,), generator=g, dtype=torch.int32)
    p, m = torch.rand(rows, generator=g) * 1.2, torch.rand(rows, generator=g) * 0.3 - 0.1
    run_rows(logits(rows, V, dtype, 7), temperature=t.cuda(), top_k=k.cuda(), top_p=p.cuda(), min_p=m.cuda())


def test_blocks_share_their_sequences_settings():
    import paper_2312_11462_amd as P
    x = logits(24, 900, torch.float32, 3).view(4, 6, 900)
    t, p = torch.tensor([0.0, 0.5, 1.0, 2.0]).cuda(), torch.tensor([0.9, 0.5, 1.0, 0.7]).cuda()
    u = torch.rand(4, 6, generator=torch.Generator().manual_seed(1)).cuda()
    tokens, probs = P.sample(x, u, temperature=t, top_p=p), P.filter_probs(x, temperature=t, top_p=p)
    assert tokens.shape == (4, 6) and probs.shape == x.shape
    flat = run_rows(x.view(24, 900), u.view(24), temperature=t.repeat_interleave(6), top_p=p.repeat_interleave(6))
    assert torch.equal(tokens.view(24), flat[0]) and torch.equal(probs.view(24, 900), flat[1])


@pytest.mark.parametrize("kw", [dict(), dict(top_k=7), dict(top_k=1000), dict(top_p=0.5), dict(top_k=900, top_p=0.37), dict(top_p=0.5, min_p=0.5), dict(temperature=0.0)], ids=str)
@pytest.mark.parametrize("V,levels", [(1000, 1), (1000, 2), (32000, 1), (32000, 3), (32000, 40), (5000, 700)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits_go_by_the_lowest_token(V, levels, dtype, kw):
    """Few distinct values: borders lie among equal tokens, more of them than are ranked one by one."""
    g = torch.Generator().manual_seed(V + levels)
    x = torch.randint(0, levels, (4, V), generator=g).float() * 0.125
    run_rows((x - 6.0).to(dtype).cuda(), **kw)
    _, probs = run_rows(x.to(dtype).cuda(), **kw)
    if levels == 1 and kw == dict(top_k=7):
        assert probs.nonzero()[:, 1].view(4, 7).tolist() == [list(range(7))] * 4


@pytest.mark.parametrize("kw", [dict(top_k=300), dict(top_k=1500, top_p=0.6), dict(top_p=0.3), dict(top_p=0.55), dict(top_p=0.9)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_crowds_around_zero(dtype, kw):
    """Hundreds of 0, -0 and of the numbers next to them on either side."""
    near = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-38, -1e-38, 1e-3, -1e-3, 1e-45, -1e-45])
    x = near[torch.randint(0, 10, (5, 6000), generator=torch.Generator().manual_seed(1))]
    x[1] = x[1] * (x[1] != 0)                                # no -0
    x[2] = -x[2].abs()                                       # no number above it
    x[3, ::2] = torch.where(x[3, ::2] == 0, torch.tensor(-0.0), x[3, ::2])
    run_rows(x.to(dtype).cuda(), **kw)


@pytest.mark.parametrize("dtype,least", [(torch.bfloat16, 2.0 ** -133), (torch.float32, 2.0 ** -149)])
def test_zero_beside_the_smallest_numbers_in_one_step(dtype, least):
    """0 and -0 are one number, though there are three between the least negative number and it; the temperature leaves just these in a step."""
    x = torch.zeros(3, 900)
    x[0, 300:600], x[0, 600:] = -least, -1.0
    x[1, ::3], x[1, 1::3] = -least, -0.0
    x[2, ::2], x[2, 1::4] = -0.0, -least
    for k in (250, 400, 700):
        run_rows(x.to(dtype).cuda(), temperature=1.3 * 64 * least, top_k=k)
    for p in (0.3, 0.55, 0.8):
        run_rows(x.to(dtype).cuda(), temperature=1.3 * 64 * least, top_p=p)


@pytest.mark.parametrize("V", [37, 1000, 40000])
def test_crowded_steps(V):
    """Logits that differ by less than a step of any histogram, all of them above one another: thousands to be told apart by their last bits."""
    base = torch.tensor(8.0).view(torch.int32)
    x = (base + torch.randperm(V, generator=torch.Generator().manual_seed(V)).int()).view(torch.float32)[None].repeat(3, 1).cuda()
    for kw in (dict(top_k=V // 3), dict(top_p=0.25), dict(top_k=V // 2, top_p=0.5), dict(temperature=100.0, top_p=0.9)):
        run_rows(x, **kw)


@pytest.mark.parametrize("kw", [dict(), dict(top_k=3), dict(top_p=0.6), dict(min_p=0.1), dict(temperature=0.0), dict(temperature=3.0, top_k=20, top_p=0.9)], ids=str)
@pytest.mark.parametrize("V", [40, 3000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logits_that_are_not_finite(V, dtype, kw):
    inf, nan = math.inf, math.nan
    x = logits(12, V, torch.float32, 5, likely=4)
    x[0, :] = -inf
    x[1, :] = nan
    x[2, :] = -inf
    x[2, 17] = -3.0e38                                       # one token left
    x[3, ::2] = -inf
    x[4, 1::2] = nan
    x[5, 5] = inf
    x[6, [3, 9, V - 1]] = inf
    x[7, :] = torch.finfo(torch.float32).min                 # masks of the lowest value: all alike
    x[8, :-1] = torch.finfo(torch.float32).min
    x[9, :] = 0.0
    x[9, ::3] = -0.0                                         # equal to 0
    x[10, :] = inf
    x[11, 4], x[11, 6] = nan, inf
    if dtype == torch.bfloat16:
        x[7, :], x[8, :-1] = torch.finfo(dtype).min, torch.finfo(dtype).min
        x[2, 17] = torch.finfo(dtype).min
    x[11, 20:30] = torch.finfo(dtype).max                    # as good as infinity
    run_rows(x.to(dtype), **kw)


@pytest.mark.parametrize("t", [0.0, 1e-38, 1e-30, 1e-3, 50.0, 1e30, math.inf])
def test_extreme_temperatures(t):
    x = logits(3, 2000, torch.float32, 9)
    for kw in (dict(), dict(top_k=11), dict(top_p=0.7), dict(min_p=0.5)):
        run_rows(x, temperature=t, **kw)


def test_temperatures_on_the_device_that_are_no_temperatures():
    """NaN and negative ones, which the host cannot see, leave the largest alone."""
    x = logits(4, 500, torch.float32, 2)
    tokens, probs = run_rows(x, temperature=torch.tensor([math.nan, -1.0, -math.inf, 0.0]).cuda())
    assert torch.equal(tokens.long(), x.argmax(-1)) and (probs.sum(-1) == 1).all()


def test_uniform_numbers_at_the_ends():
    import paper_2312_11462_amd as P
    x = logits(1, 3000, torch.float32, 4).repeat(6, 1)
    u = torch.tensor([0.0, 2.0 ** -149, 1 - 2.0 ** -24, 1.0, -1.0, 2.0]).cuda()
    tokens, probs = run_rows(x, u, top_p=0.8)
    stay = probs[0].nonzero()[:, 0]
    assert tokens.tolist() == [stay[0], stay[0], stay[-1], stay[-1], stay[0], stay[-1]]
    assert 0 <= P.sample(x[:1], torch.tensor([math.nan]).cuda()).item() < 3000


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 0x7F800001), (torch.float32, -0x7FFFFF), (torch.float32, 0x7FC00000), (torch.bfloat16, 0x7F81), (torch.bfloat16, -0x7F)])
def test_every_kind_of_nan(dtype, bits):
    for V in (1, 300, 5000):
        x = logits(4, V, dtype, 3)
        raw = x.view(torch.int32 if dtype == torch.float32 else torch.int16)
        raw[0, :] = bits
        raw[1, ::2] = bits
        raw[2, V // 2:] = bits
        for kw in (dict(), dict(top_k=5), dict(top_p=0.7), dict(min_p=0.1), dict(temperature=0.0)):
            run_rows(x, **kw)


def test_values_far_apart():
    x = torch.tensor([[3.0e38, -3.0e38, 3.0e38, 1.0], [1e-40, 0.0, -1e-40, 1e-44], [88.0, 87.9, -104.0, 20.0]]).cuda()
    for kw in (dict(), dict(top_k=2), dict(top_p=0.5), dict(temperature=1e-40), dict(min_p=0.95)):
        run_rows(x, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad,shift", [(1000, 1, 0), (1001, 0, 1), (32000, 128, 3), (32001, 3, 5), (7, 2, 1)])
def test_rows_of_any_alignment_inside_a_wider_buffer(V, pad, shift, dtype):
    """What lies between the rows is larger than any logit."""
    rows = 4
    wide = torch.full((shift + rows * (V + pad) + 8,), 1e4, dtype=dtype, device="cuda")
    x = wide[shift:shift + rows * (V + pad)].view(rows, V + pad)[:, :V]
    x.copy_(logits(rows, V, dtype, V))
    assert x.stride(0) == V + pad
    dense = x.contiguous()
    u = torch.rand(rows, generator=torch.Generator().manual_seed(2)).cuda()
    for kw in (dict(top_k=5), dict(top_p=0.9, min_p=0.001)):
        a, b = run_rows(x, u, **kw), run_rows(dense, u, **kw)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_outputs_end_where_they_end():
    import paper_2312_11462_amd as P
    x = logits(3, 1001, torch.float32, 1)
    room = torch.full((3 * 1001 + 16,), 7.0, device="cuda")
    P.filter_probs(x, top_p=0.9, out=room[8:8 + 3 * 1001].view(3, 1001))
    assert (room[:8] == 7).all() and (room[-8:] == 7).all()
    ids = torch.full((5,), 9, dtype=torch.int32, device="cuda")
    P.sample(x, torch.rand(3).cuda(), out=ids[1:4])
    assert ids[0] == 9 and ids[4] == 9 and (ids[1:4] >= 0).all() and (ids[1:4] < 1001).all()
    assert P.filter_probs(x[:0]).shape == (0, 1001) and P.sample(x[:0], torch.rand(0).cuda()).shape == (0,)


def test_draws_follow_the_probabilities():
    """One row, an even grid of uniform numbers: every token is drawn as often as its probability says, to one step of the grid at either end."""
    import paper_2312_11462_amd as P
    n = 1 << 14
    x = logits(1, 300, torch.float32, 8)
    probs = P.filter_probs(x, temperature=0.9, top_k=30, top_p=0.95)[0].double().cpu()
    tokens = P.sample(x.expand(n, 300).contiguous(), torch.arange(n).float().cuda() / n, temperature=0.9, top_k=30, top_p=0.95)
    count = torch.bincount(tokens.long().cpu(), minlength=300).double()
    assert (tokens[1:] >= tokens[:-1]).all() and ((count - n * probs).abs() <= 1 + n * 300 * 2.0 ** -23).all()


def test_a_review_with_filtered_rows_keeps_drafts_of_the_same_filter():
    """Drafts drawn from q and reviewed against p = q are always kept; the extra token is one that stays."""
    import paper_2312_11462_amd as P
    B, k, V = 3, 4, 1200
    x = logits(B * (k + 1), V, torch.float32, 6).view(B, k + 1, V)
    t = torch.tensor([0.7, 1.0, 1.3]).cuda()
    u = torch.rand(B, k + 1, generator=torch.Generator().manual_seed(3)).cuda()
    p = P.filter_probs(x, temperature=t, top_k=25, top_p=0.9)
    draft = P.sample(x, u, temperature=t, top_k=25, top_p=0.9)[:, :k].contiguous()
    n, nxt = P.accept(p, p[:, :k].contiguous(), draft, u[:, :k].contiguous(), u[:, k].contiguous())
    assert n.tolist() == [k] * B and all(p[b, k, nxt[b]] > 0 for b in range(B))


# ------------------------------------------------------------------------------------------------ pages

class Both:
    """The arrays on the GPU, and the oracle's."""

    def __init__(self, n_pages, page, sequences, entries, seed=0):
        import paper_2312_11462_amd as P
        self.rng = np.random.default_rng(seed)
        self.gpu = P.Pages.new(n_pages, page, sequences, entries)
        order = self.rng.permutation(n_pages).astype(np.int32)
        self.gpu.free.copy_(torch.tensor(order))
        self.ref = O.Pages(self.gpu.table.tolist(), self.gpu.held.tolist(), order, [0] * n_pages, page)

    def dev(self, x):
        return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")

    def same(self):
        n = int(self.gpu.n_free)
        assert self.gpu.table.tolist() == self.ref.table and self.gpu.held.tolist() == self.ref.held
        assert n == len(self.ref.free) and self.gpu.free[:n].tolist() == self.ref.free and self.gpu.users.tolist() == self.ref.users

    def plan(self, cache_len, new_rows, rows):
        got = self.gpu.plan(self.dev(cache_len), self.dev(new_rows), rows)
        want = self.ref.plan(cache_len, new_rows, rows)
        for g, w, name in zip(got, want, ("row_start", "sequence", "position", "slot", "served")):
            assert g.tolist() == w, name
        self.same()
        return want

    def release(self, keep):
        self.gpu.release(self.dev(keep))
        self.ref.release(keep)
        self.same()

    def share(self, source, length):
        self.gpu.share(self.dev(source), self.dev(length))
        self.ref.share(source, length)
        self.same()


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("sequences", [1, 7, 64, 1500])
def test_sequences_come_grow_and_go(sequences, page):
    """Twelve steps of a server: prompts enter, blocks are reviewed and cut, sequences end, prompts are shared; pages run out on the way."""
    entries = 12
    c = Both(max(4, sequences * 4), page, sequences, entries, seed=sequences + page)
    length = np.zeros(sequences, dtype=np.int64)
    for step in range(12):
        new = np.where(c.rng.random(sequences) < 0.2, c.rng.integers(0, 3 * page, sequences), c.rng.integers(0, 6, sequences))
        if step % 4 == 2:
            new[c.rng.integers(sequences)] = 13 * page       # more than a table holds
        rows = int(new.sum()) if step % 3 else int(new.sum()) * 3 // 4
        served = c.plan(length, new, rows)[4]
        length = np.where(served, length + c.rng.integers(0, new + 1), length)
        length[c.rng.random(sequences) < 0.15] = 0
        keep = np.where(c.rng.random(sequences) < 0.2, -1, length)
        c.release(keep)
        if step % 2:
            source = np.where(c.rng.random(sequences) < 0.3, c.rng.integers(-1, sequences + 1, sequences), -1)
            at = c.rng.integers(0, 5 * page, sequences)
            held = np.array(c.ref.held)
            c.share(source, at)
            length = np.where((held == 0) & (np.array(c.ref.held) > 0), np.array(c.ref.held) * page, length)
    c.release(np.zeros(sequences, dtype=np.int64))
    assert int(c.gpu.n_free) == c.ref.n_pages and not c.gpu.users.any()


def test_long_prompts_and_thousands_of_rows():
    c = Both(2000, 16, 40, 600, seed=3)
    new = [5000, 1, 0, 9000, 4097] + [1] * 35
    c.plan([0] * 40, new, sum(new) + 100)
    c.release([0, -1, -1, 8999, 4096] + [-1] * 35)
    c.plan([0, 1, 0, 8999, 4096] + [1] * 35, [17] * 40, 17 * 40)


def test_the_same_page_is_given_up_by_many_in_one_call():
    c = Both(64, 16, 30, 4, seed=5)
    c.plan([0] * 30, [50] + [0] * 29, 50)
    c.share([-1] + [0] * 20 + [-1] * 9, [0] + [48] * 20 + [0] * 9)
    assert max(c.ref.users) == 21
    c.release([-1] + [0] * 10 + [16] * 10 + [-1] * 9)
    c.release([0] * 30)
    assert c.ref.free[-1] == c.gpu.free[63].item()


def test_pages_without_enough_left_serve_the_first_and_those_who_need_none():
    c = Both(4, 16, 5, 8, seed=1)
    assert c.plan([0] * 5, [20, 20, 20, 0, 1], 64)[4] == [1, 1, 0, 1, 0]
    assert c.plan([20, 20, 0, 0, 0], [5, 12, 0, 0, 16], 64)[4] == [1, 1, 1, 1, 0]
    assert c.plan([25, 32, 0, 0, 0], [1, 1, 0, 0, 0], 1)[4] == [1, 0, 1, 1, 1]      # a row too many


def test_entries_that_name_no_page_are_passed_over():
    """A caller that has given pages back by itself (a sliding window): their entries are -1."""
    c = Both(32, 16, 3, 8, seed=2)
    c.plan([0, 0, 0], [100, 40, 0], 140)
    for b, i in ((0, 0), (0, 1), (1, 0)):
        page = c.ref.table[b][i]
        c.ref.table[b][i] = -1
        c.gpu.table[b, i] = -1
        c.ref.users[page] = 0
        c.gpu.users[page] = 0
        c.ref.free.append(page)
        c.gpu.free[int(c.gpu.n_free)] = page
        c.gpu.n_free += 1
    c.plan([100, 5, 0], [3, 2, 0], 5)
    c.share([-1, -1, 0], [0, 0, 64])
    c.release([10, 0, -1])


def test_lengths_that_are_no_lengths():
    c = Both(16, 16, 4, 4)
    c.plan([-5, 0, 2 ** 31 - 1, 1], [3, -7, 2 ** 31 - 1, 20], 40)
    c.release([-2 ** 31, 0, 2 ** 31 - 1, 1])


def test_no_rows_in_a_step():
    c = Both(16, 16, 4, 4)
    assert c.plan([0] * 4, [0] * 4, 0)[0] == [0] * 5


# ------------------------------------------------------------------------------------------------ cross-attention

class States(Paged):
    """Encoder states in pages; the rows of a call are in none."""

    def __init__(self, cache, rows, length, new, **kw):
        super().__init__(cache, rows, length, [0] * len(length), **kw)
        self.new = list(new)
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.total = int(self.start[-1])
        self.dev[1] = torch.tensor(self.start, device="cuda")
        start = torch.tensor(np.concatenate([[0], np.cumsum(length)]), dtype=torch.int32, device="cuda")
        if sum(length):
            self.kv.write(0, self.dev[0], start, torch.zeros(len(length), dtype=torch.int32, device="cuda"), self.random_rows(sum(length)),
                          self.random_rows(sum(length), loud=False))

    def cross(self, q, scale, max_rows=None, **kw):
        return self.kv.cross_attention(0, *self.dev, q, scale, max_rows, **kw)

    def check_cross(self, out, q, scale):
        # the bound of the module next door (test_gpu_paged), with as many keys as the longest encoder has
        k, v = self.values(self.k, self.ks)[0], self.values(self.v, self.vs)[0]
        qq = q.double().cpu().numpy()
        want = O.cross_attention(k, v, self.table, self.start, self.cached, qq, scale)
        size = O.cross_attention(k, np.abs(v), self.table, self.start, self.cached, qq, scale)
        live = k[np.isfinite(k).all(-1)]
        dot = abs(scale) * np.sqrt((qq ** 2).sum(-1)).max(initial=0) * np.sqrt((live ** 2).sum(-1)).max(initial=0)
        e = (self.d + 4) * 2.0 ** -24 * dot + 2.0 ** -21 + max(self.cached) * 2.0 ** -24
        bf = self.rows == "bf16"
        tol = (2.0 ** -8 if bf else 2.0 ** -24) * np.abs(want) + 2 * ((2.0 ** -8 if bf else 0.0) + e) * size
        got = out.double().cpu().numpy()[:self.total]
        want, tol = want[:self.total], tol[:self.total]
        assert np.array_equal(np.isfinite(got), np.isfinite(want))
        fine = np.isfinite(want)
        err = np.abs(got - want)[fine]
        assert (err <= tol[fine]).all(), f"off by {(err / np.maximum(tol[fine], 1e-300)).max():.2f} times the bound"


TYPES = [("fp32", "fp32"), ("fp32", "bf16"), ("fp32", "fp8"), ("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "fp32")]


@pytest.mark.parametrize("d,kv_heads,group", [(16, 2, 1), (64, 4, 1), (64, 2, 8), (80, 1, 3), (128, 2, 4), (256, 1, 1)])
@pytest.mark.parametrize("rows,cache", TYPES)
def test_cross_attention_of_ragged_batches(rows, cache, d, kv_heads, group):
    """Encoders of no row, one, a page and more; blocks, single tokens and a sequence without rows."""
    c = States(cache, rows, [0, 1, 16, 17, 300, 0, 45], [3, 5, 1, 2, 4, 1, 0], kv_heads=kv_heads, group=group, d=d, width=2, seed=d + group)
    q = c.random_rows(c.total, heads=kv_heads * group)
    for most in (None, max(c.new)):
        out = c.cross(q, d ** -0.5, most)
        c.check_cross(out, q, d ** -0.5)
        assert not out[:3].any() and not out[15:16].any()


@pytest.mark.parametrize("rows,cache,d", [("bf16", "bf16", 64), ("bf16", "fp8", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 128), ("fp32", "fp32", 64)])
@pytest.mark.parametrize("length,new", [([700, 0, 63], [40, 1, 64]), ([64, 1000], [33, 70]), ([129, 300, 0, 65], [200, 1, 1, 130]), ([0, 513], [300, 5])], ids=str)
def test_cross_attention_of_blocks_and_chunks(rows, cache, d, length, new):
    """Every kernel, with an encoder that has no row among the long ones."""
    c = States(cache, rows, length, new, kv_heads=2, group=2, d=d, page=32, seed=len(new))
    q = c.random_rows(c.total, heads=4)
    c.check_cross(c.cross(q, d ** -0.5, max(new)), q, d ** -0.5)


@pytest.mark.parametrize("cache,d", [("bf16", 64), ("fp8", 128)])
@pytest.mark.parametrize("many", [False, True])
def test_cross_attention_of_prompts_that_fill_the_chip(cache, d, many):
    """More items than are shared out: a workgroup for each; some encoders have no row, one row, or as many as another.  many: more sequences than a wave has lanes."""
    if many:
        length, new, kv_heads = [(37 * b) % 150 for b in range(70)], [400 - b % 7 for b in range(70)], 4
    else:
        length, new, kv_heads = [90, 0, 1, 200, 65, 200], [300, 257, 400, 260, 300, 290], 96
    c = States(cache, "bf16", length, new, kv_heads=kv_heads, group=2, d=d, page=16, seed=d)
    q = c.random_rows(c.total, heads=2 * kv_heads)
    out = c.cross(q, d ** -0.5, max(new))
    k, v = c.values(c.k, c.ks)[0][:, :2], c.values(c.v, c.vs)[0][:, :2]
    for r in np.unique(np.concatenate([c.start[:-1], c.start[1:] - 1, c.start[:-1] + 256])):         # (the first two key-value heads, rows at the ends of sequences and row tiles)
        b = int(np.searchsorted(c.start, r, side="right")) - 1
        one = q[r:r + 1, :4].double().cpu().numpy()
        want = O.cross_attention(k, v, c.table[b:b + 1], [0, 1], [length[b]], one, d ** -0.5)
        size = O.cross_attention(k, np.abs(v), c.table[b:b + 1], [0, 1], [length[b]], one, d ** -0.5)
        got = out[r:r + 1, :4].double().cpu().numpy()
        # scores of |q| |k| below 40 here: their error is far below a weight's rounding to bf16
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2 * (2.0 ** -8 + 2.0 ** -12) * size).all(), r


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_long_encoders_shared_out_over_the_chip(cache):
    c = States(cache, "bf16", [9000, 0, 4097, 1], [5, 2, 1, 3], kv_heads=2, group=1, d=64, page=64, seed=8)
    q = c.random_rows(c.total, heads=2)
    c.check_cross(c.cross(q, 0.125, 5), q, 0.125)


@pytest.mark.parametrize("rows,cache,d", [("bf16", "bf16", 64), ("bf16", "fp8", 128), ("fp32", "fp32", 32)])
def test_single_tokens_attend_as_attention_does(rows, cache, d):
    """One row per sequence at the last of t + 1 positions attends them all: the same keys, the same bits."""
    c = States(cache, rows, [1, 40, 700, 33], [1, 1, 1, 1], kv_heads=2, group=4, d=d, seed=4)
    q = c.random_rows(4, heads=8)
    last = torch.tensor([n - 1 for n in c.cached], dtype=torch.int32, device="cuda")
    assert torch.equal(c.cross(q, d ** -0.5, 1), c.kv.attention(0, c.dev[0], c.dev[1], last, q, d ** -0.5, 1))


@pytest.mark.parametrize("rows,cache,d,m", [("bf16", "bf16", 64, 5), ("bf16", "fp8", 128, 40), ("fp32", "fp32", 16, 3), ("bf16", "bf16", 128, 200)])
def test_encoder_rows_without_a_page_and_lengths_beyond_the_table(rows, cache, d, m):
    c = States(cache, rows, [100, 64, 48, 30], [m, 2, m, 1], kv_heads=2, d=d, seed=6)
    c.table[0, [1, 3]] = -1
    c.table[1, :] = -1                                       # nothing left
    c.table[2, 1] = c.n_pages + 7                            # no page either
    c.dev[0] = torch.tensor(c.table, device="cuda")
    c.cached = [100, 64, 48, c.table.shape[1] * 16]
    c.table[3, 2:] = -1
    c.dev[0] = torch.tensor(c.table, device="cuda")
    c.dev[2] = torch.tensor([100, 64, 48, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    # (positions 30 and 31 of the last sequence are in its second page, and were never written)
    for x in (c.k, c.v):
        raw = x.view(torch.uint8)
        raw[0, int(c.table[3, 1]), :, 14:] = 0
    if c.ks is not None:
        c.ks[0, int(c.table[3, 1]), :, 14:] = 127
        c.vs[0, int(c.table[3, 1]), :, 14:] = 127
    q = c.random_rows(c.total, heads=2)
    out = c.cross(q, d ** -0.5, m)
    c.check_cross(out, q, d ** -0.5)
    assert not out[m:m + 2].any()


@pytest.mark.parametrize("rows,cache,d,m", [("bf16", "bf16", 64, 3), ("bf16", "fp8", 64, 70), ("fp32", "bf16", 64, 2)])
def test_rows_inside_a_wider_buffer_and_rows_of_no_sequence(rows, cache, d, m):
    c = States(cache, rows, [50, 20], [m, m], kv_heads=2, d=d, seed=7)
    wide = torch.full((c.total + 5, 3, 2, d), 9.0, dtype=c.random_rows(1).dtype, device="cuda")
    q = wide[:, 1]
    q[2:2 + c.total] = c.random_rows(c.total, heads=2)
    start = c.dev[1] + 2
    out = torch.full((c.total + 5, 2, d), 3.0, dtype=wide.dtype, device="cuda")
    got = c.kv.cross_attention(0, c.dev[0], start, c.dev[2], q, 0.125, m, out=out)
    assert got is out and (out[:2] == 3).all() and (out[2 + c.total:] == 3).all()
    c.check_cross(out[2:2 + c.total], q[2:2 + c.total], 0.125)
    longer = c.kv.cross_attention(0, c.dev[0], start, c.dev[2], q, 0.125, 1, out=torch.full_like(out, 3.0))
    assert (longer[3:2 + m] == 3).all() and torch.isfinite(longer).all()                 # (cut to one row each: the others are left)


@pytest.mark.parametrize("rows,cache,d,m", [("bf16", "bf16", 64, 2), ("bf16", "bf16", 128, 50), ("fp32", "fp32", 64, 2), ("bf16", "bf16", 128, 300)])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_values_behind_the_encoders_last_row_reach_nobody(rows, cache, d, m, what):
    c = States(cache, rows, [37, 5], [m, m], kv_heads=2, d=d, seed=9)
    c.k[0, c.table[0, 2], :, 37 % 16:] = what
    c.v[0, c.table[0, 2], :, 37 % 16:] = what
    c.v[0, c.table[1, 0], :, 5:] = -what
    q = c.random_rows(c.total, heads=2)
    out = c.cross(q, d ** -0.5, m)
    assert torch.isfinite(out).all()
    clean = States(cache, rows, [37, 5], [m, m], kv_heads=2, d=d, seed=9, poison=False)
    assert torch.equal(out, clean.cross(q, d ** -0.5, m))


@pytest.mark.parametrize("scale", [1.0, -0.3, 0.0])
def test_scales(scale):
    for rows, cache, d, m in (("bf16", "fp8", 64, 4), ("bf16", "bf16", 128, 90), ("fp32", "fp32", 16, 2)):
        c = States(cache, rows, [200, 3], [m, m], kv_heads=1, group=2, d=d, seed=3)
        q = 0.2 * c.random_rows(c.total, heads=2)
        c.check_cross(c.cross(q, scale, m), q, scale)


# ------------------------------------------------------------------------------------------------ together

def step_of_a_server(P, kv, cross_kv, pages, enc_table, enc_len, length, new, rows, most, w, u, limits):
    """Plan, write, attend the sequence and the encoder, draw: one step in which every sequence gets new[b] rows.  Returns (row_start, tokens, probabilities)."""
    row_start, seq, pos, slot, served = pages.plan(length, new, rows)
    table = pages.table
    heads, d = kv.n_kv_heads, kv.head_dim
    x = w["embed"][(pos.clamp(min=0) * 7 + seq.clamp(min=0)).long() % w["embed"].shape[0]]          # [rows][heads * d]
    q, k, v = ((x @ w[n]).view(rows, heads, d).to(torch.bfloat16) for n in ("q", "k", "v"))
    kv.write(0, table, row_start, length, k, v)
    h = kv.attention(0, table, row_start, length, q, d ** -0.5, most)
    h = cross_kv.cross_attention(0, enc_table, row_start, enc_len, h, 1.0, most)
    out = h.view(rows, heads * d).float() @ w["head"]
    probs = torch.empty(out.shape, device="cuda")
    tokens = P.sample(out, u, temperature=0.8, top_k=limits[0], top_p=limits[1], probs=probs)
    return row_start, seq, pos, slot, served, q, k, v, h, out, tokens, probs


def test_a_step_of_a_server():
    """Prompts enter, then blocks of four drafts are scored, cut and scored again, over pages that the plan deals out; every intermediate result against the plain forms."""
    import paper_2312_11462_amd as P
    B, heads, d, V, page = 5, 2, 64, 777, 16
    g = torch.Generator(device="cuda").manual_seed(11)
    w = {n: torch.randn(heads * d, heads * d, generator=g, device="cuda") * 0.09 for n in ("q", "k", "v")}
    w["embed"], w["head"] = torch.randn(97, heads * d, generator=g, device="cuda"), torch.randn(heads * d, V, generator=g, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    kv = P.PagedKv(*(torch.zeros(1, 24, heads, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    pages = P.Pages.new(24, page, B, 8)
    ref = O.Pages(pages.table.tolist(), [0] * B, pages.free.tolist(), [0] * 24, page)
    enc = P.PagedKv(*(torch.zeros(1, 12, heads, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    enc_pages = P.Pages.new(12, page, B, 4)
    enc_len = torch.tensor([20, 0, 33, 16, 1], **i32)
    enc_start, *_ = enc_pages.plan(torch.zeros(B, **i32), enc_len, 70)
    enc.write(0, enc_pages.table, enc_start, torch.zeros(B, **i32), *(torch.randn(70, heads, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)))
    length = torch.zeros(B, **i32)
    for step, (new, keep) in enumerate([([30, 17, 1, 40, 5], [30, 17, 1, 40, 5]), ([5, 5, 5, 5, 5], [32, 20, 6, 41, 7]), ([5, 5, 0, 5, 5], [33, 25, 0, 42, 8])]):
        rows = sum(new)
        u = torch.rand(rows, generator=g, device="cuda")
        row_start, seq, pos, slot, served, q, k, v, h, out, tokens, probs = step_of_a_server(
            P, kv, enc, pages, enc_pages.table, enc_len, length, torch.tensor(new, **i32), rows, max(new), w, u, (40, 0.9))
        want = ref.plan(length.tolist(), new, rows)
        assert [x.tolist() for x in (row_start, seq, pos, slot, served)] == list(want) and pages.table.tolist() == ref.table
        # the rows lie where the plan says
        assert torch.equal(kv.k[0].transpose(1, 2).reshape(-1, heads, d)[slot], k)
        def host(x):
            return x.double().cpu().numpy()
        from oracle import paged as OP
        a = OP.attention(host(kv.k[0]), host(kv.v[0]), np.array(ref.table), want[0], length.tolist(), host(q), d ** -0.5)
        # (the attention's own output is bf16 and the queries of the next one: taken from the GPU by a call of its own)
        mid = kv.attention(0, pages.table, row_start, length, q, d ** -0.5, max(new))
        assert np.abs(host(mid) - a).max() <= 3 * 2.0 ** -8 * np.abs(host(kv.v[0])).max()
        c = O.cross_attention(host(enc.k[0]), host(enc.v[0]), enc_pages.table.cpu().numpy(), want[0], enc_len.tolist(), host(mid), 1.0)
        assert np.abs(host(h) - c).max() <= 3 * 2.0 ** -8 * np.abs(host(enc.v[0])).max()
        check_rows(host(out), tokens.cpu().numpy(), probs.cpu().numpy(), u.cpu().numpy(), as_sets(rows, 0.8, 40, 0.9, 0.0))
        pages.release(torch.tensor(keep, **i32))
        ref.release(keep)
        assert pages.table.tolist() == ref.table and pages.users.tolist() == ref.users
        length = torch.tensor(keep, **i32)


def test_a_captured_step_replays_to_the_eager_result():
    """One graph of a whole step; between replays the lengths move on and eager work runs.  Every replay is checked against the same step run eagerly from the same state."""
    import paper_2312_11462_amd as P
    B, heads, d, V, page = 4, 2, 64, 500, 16
    g = torch.Generator(device="cuda").manual_seed(12)
    w = {n: torch.randn(heads * d, heads * d, generator=g, device="cuda") * 0.09 for n in ("q", "k", "v")}
    w["embed"], w["head"] = torch.randn(97, heads * d, generator=g, device="cuda"), torch.randn(heads * d, V, generator=g, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    kv = P.PagedKv(*(torch.zeros(1, 40, heads, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    enc = P.PagedKv(*(torch.randn(1, 12, heads, page, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)))
    enc_table, enc_len = torch.arange(12, **i32).view(4, 3), torch.tensor([48, 0, 7, 30], **i32)
    pages = P.Pages.new(40, page, B, 10)
    length, new, u = torch.zeros(B, **i32), torch.full((B,), 5, **i32), torch.rand(20, generator=g, device="cuda")
    keep = torch.zeros(B, **i32)

    def step():
        out = step_of_a_server(P, kv, enc, pages, enc_table, enc_len, length, new, 20, 5, w, u, (30, 0.95))
        pages.release(keep)
        return out
    state = (kv.k, kv.v, pages.table, pages.held, pages.free, pages.n_free, pages.users)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        length.copy_(torch.tensor([7 * i, 3 * i, 16 * i, i]))
        pages.plan(length, torch.zeros(B, **i32), 0)
        keep.copy_(length)
        u.copy_(torch.rand(20, generator=g, device="cuda"))
        before = [x.clone() for x in state]
        graph.replay()
        got = [x.clone() for x in captured] + [x.clone() for x in state]
        torch.cuda.synchronize()
        for x, y in zip(state, before):
            x.copy_(y)
        eager = list(step()) + [x.clone() for x in state]
        for a, b in zip(got, eager):
            assert torch.equal(a, b), i


def test_calls_on_another_stream_follow_that_stream():
    import paper_2312_11462_amd as P
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    x = torch.zeros(4, 32000, device="cuda")
    fresh = logits(4, 32000, torch.float32, 5)
    u = torch.rand(4, generator=torch.Generator().manual_seed(4)).cuda()
    want = P.sample(fresh, u, top_p=0.9), P.filter_probs(fresh, top_k=9)
    pages = P.Pages.new(64, 16, 8, 8)
    length, new = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            big = (big @ big).clamp(-1, 1)
        x.copy_(fresh)
        new.fill_(33)
        got = P.sample(x, u, top_p=0.9), P.filter_probs(x, top_k=9)
        plan = pages.plan(length, new, 300)
        pages.release(length)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert plan[0].tolist() == [33 * b for b in range(9)] and int(pages.n_free) == 64


def test_threads_that_draw_at_once():
    import threading

    import paper_2312_11462_amd as P
    x = [logits(20, 5000, torch.float32, i) for i in range(4)]
    u = torch.rand(20, generator=torch.Generator().manual_seed(6)).cuda()
    want = [P.sample(a, u, top_k=i + 2, top_p=0.9) for i, a in enumerate(x)]
    bad = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
            for _ in range(50):
                got = P.sample(x[i], u, top_k=i + 2, top_p=0.9)
                torch.cuda.current_stream().synchronize()
                if not torch.equal(got, want[i]):
                    bad.append(i)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_refusals_of_the_binding():
    import paper_2312_11462_amd as P
    x, u = logits(6, 50, torch.float32), torch.rand(6).cuda()
    for bad in (dict(temperature=torch.ones(6)), dict(temperature=torch.ones(4).cuda()), dict(top_p=torch.ones(6).cuda(), min_p=torch.ones(3).cuda()),
                dict(top_p=torch.ones(12).cuda()[::2])):
        with pytest.raises(ValueError):
            P.sample(x, u, **bad)
    for bad in (dict(temperature=torch.ones(6).double().cuda()), dict(top_k=torch.ones(6).long().cuda())):
        with pytest.raises(TypeError):
            P.filter_probs(x, **bad)
    for bad in (dict(temperature=-1.0), dict(top_p=math.nan), dict(min_p=2.0)):
        with pytest.raises(P.CsdError):
            P.filter_probs(x, **bad)
    with pytest.raises(TypeError):
        P.sample(x.double(), u)
    with pytest.raises(TypeError):
        P.sample(x, u.double())
    with pytest.raises(ValueError):
        P.sample(x, u[:5])
    with pytest.raises(ValueError):
        P.sample(x.t(), torch.rand(50).cuda())
    with pytest.raises(ValueError):
        P.sample(x.view(2, 3, 50).transpose(0, 1), torch.rand(3, 2).cuda())
    with pytest.raises(ValueError):
        P.filter_probs(x, out=torch.empty(6, 51, device="cuda"))
    with pytest.raises(ValueError):
        P.sample(x, u, probs=torch.empty(50, 6, device="cuda").t())
    pages = P.Pages.new(8, 16, 3, 2)
    n = torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (n.cpu(), n[:2], torch.zeros(6, dtype=torch.int32, device="cuda")[::2]):
        with pytest.raises(ValueError):
            pages.plan(bad, n, 4)
        with pytest.raises(ValueError):
            pages.release(bad)
        with pytest.raises(ValueError):
            pages.share(n, bad)
    with pytest.raises(TypeError):
        pages.plan(n, n.long(), 4)
    with pytest.raises(P.CsdError):
        P.Pages(pages.table, pages.held, pages.free, pages.n_free, pages.users, 24).release(n)
    c = States("bf16", "bf16", [20], [3], seed=1)
    q = c.random_rows(3, heads=2)
    with pytest.raises(ValueError):
        c.kv.cross_attention(0, c.dev[0], c.dev[1], c.dev[2].cpu(), q, 0.1)
    with pytest.raises(TypeError):
        c.kv.cross_attention(0, c.dev[0], c.dev[1], c.dev[2].long(), q, 0.1)
    with pytest.raises(ValueError):
        c.kv.cross_attention(0, c.dev[0], c.dev[1], c.dev[2], q[:, :, :32], 0.1)
    with pytest.raises(P.CsdError):
        c.kv.cross_attention(0, c.dev[0], c.dev[1], c.dev[2], q, math.nan)


def test_no_rows_of_logits_are_no_tokens():
    import paper_2312_11462_amd as P
    for shape in ((0, 64), (2, 0, 64), (0, 3, 64)):
        x = torch.empty(shape, device="cuda")
        t = P.sample(x, torch.empty(shape[:-1], device="cuda"), top_k=3)
        assert t.shape == shape[:-1] and t.dtype is torch.int32
        assert P.filter_probs(x, top_p=0.5).shape == shape


def test_offsets_beyond_32_bits():
    """Rows, distances between rows, probabilities and slots behind the 2^31st element."""
    import paper_2312_11462_amd as P
    V = 131072
    rows = (1 << 31) // V + 3
    few = logits(3, V, torch.bfloat16, 21)
    u = torch.full((rows,), 0.37, device="cuda")
    at = [0, rows - 2, rows - 1]
    want = P.sample(few, u[:3], top_p=0.9), P.filter_probs(few, top_p=0.9)
    x = torch.full((rows, V), -math.inf, dtype=torch.bfloat16, device="cuda")
    x[at] = few
    probs = torch.full((rows, V), -1.0, device="cuda")
    tokens = P.sample(x, u, top_p=0.9, probs=probs)
    assert torch.equal(tokens[at], want[0]) and torch.equal(probs[at], want[1])
    assert int((tokens == -1).sum()) == rows - 3 and not probs[1:rows - 2].any()
    far = x.flatten()[:V * (rows - 1)].as_strided((2, V), (V * (rows - 2), 1))
    assert torch.equal(P.sample(far, u[:2], top_p=0.9), want[0][:2])
    del x, probs, far
    n, i32 = 3 << 20, dict(dtype=torch.int32, device="cuda")
    pages = P.Pages(torch.full((2, 4), -1, **i32), torch.zeros(2, **i32), torch.arange(n, **i32), torch.full((1,), n, **i32), torch.zeros(n, **i32), 1024)
    _, sequence, position, slot, served = pages.plan(torch.tensor([5, 1024], **i32), torch.tensor([2, 1], **i32), 4)
    assert sequence.tolist() == [0, 0, 1, -1] and position.tolist() == [5, 6, 1024, -1] and served.tolist() == [1, 1]
    assert slot.tolist() == [(n - 1) * 1024 + 5, (n - 1) * 1024 + 6, (n - 3) * 1024, -1]
