"""The calls of a serving step where they could go wrong: chunks over tables that their lengths pass, sequences cut inside pages that others use, thousands of
sequences, rows of equal logits, borders among tokens of equal weight.  The plain forms are oracle/serving.py's; the bounds are test_gpu_serving's."""
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import Paged
from test_gpu_serving import Both, States

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
