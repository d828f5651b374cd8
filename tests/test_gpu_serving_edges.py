"""The calls of a serving step where they could go wrong: chunks over tables that their lengths pass, sequences cut inside pages that others use, thousands of
sequences, rows of equal logits, borders among tokens of equal weight.  The plain forms are oracle/serving.py's; the bounds are test_gpu_serving's."""
import math

import numpy as np
import pytest
import torch

from test_gpu_paged import Paged
from test_gpu_serving import States

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
