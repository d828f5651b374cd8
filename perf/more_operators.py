"""The operators of a serving step around the paged cache and the review: what is measured, in which sizes, and what each computes in plain form.

Kinds of case (`case["kind"]`):
  sample   tokens from logits by temperature, top-k, top-p and min-p, with uniform numbers that the caller gives
  filter   the probabilities that such a draw has, dense rows as the review of drafts takes them
  pages    the pages, row starts and slots of a step's new rows from the requests' lengths, and the pages of rows that are not kept given back
  cross    the rows of a block or chunk attend an encoder's states of another length, in pages

A row's tokens are ranked by logit, of equal ones the lowest first.  With w = exp((logit - largest) / temperature), the first top_k of the ranking
stay, of these the shortest start whose weights reach top_p of theirs, of these those with w >= min_p; the token drawn by u is the
lowest one at which the running sum of the remaining weights, by token, passes u times all of them.  A temperature of 0 leaves the largest alone.
"""
import random
from types import SimpleNamespace

import torch

own = False

_TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
_SIZE = {"fp32": 4, "bf16": 2, "fp8": 1}


def _named(c, name):
    return dict(c, name=name) if name else c


def _logits(kind, dtype, rows, vocab, by, pad=0, each=1, name=""):
    return _named(dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab, by=by, pad=pad, each=each), name)


def _pages(batch, page, lo, hi, chunk, few=0, name=""):
    return _named(dict(kind="pages", batch=batch, page=page, lo=lo, hi=hi, chunk=chunk, few=few), name)


def _cross(cache, batch, kv_heads, group, head_dim, page, lo, hi, chunk, few=0, rows="bf16", name=""):
    return _named(dict(kind="cross", rows=rows, cache=cache, batch=batch, kv_heads=kv_heads, group=group, head_dim=head_dim, page=page, lo=lo, hi=hi,
                       chunk=chunk, few=few), name)


def listed():
    """by: which of the parameters are set (mixed: another set for every sequence, greedy ones among them); pad: logits between two rows that belong to
    no token; each: rows that share a sequence's parameters; lo, hi: shortest and longest cached or encoded length; chunk: new rows of a sequence;
    few: so many sequences of the batch have one new row instead; group: query heads per key-value head."""
    return [
        # the tiny model draws one token: nothing but latency
        _logits("sample", "fp32", 1, 512, "top_k", name="sample_tiny"),
        # the draft level draws the next token of one sequence
        _logits("sample", "fp32", 1, 32000, "both", name="sample_draft"),
        # 64 sequences draw a token each, everyone with settings of their own; logits as they leave a head padded to whole tiles
        _logits("sample", "fp32", 64, 32000, "mixed", pad=128, name="sample_batch"),
        # a large vocabulary, a large batch, half precision: many logits are equal
        _logits("sample", "bf16", 256, 131072, "top_p", name="sample_wide_bf16"),
        # the review of four drafts of one sequence: five rows
        _logits("filter", "fp32", 5, 32000, "top_p", each=5, name="filter_block"),
        # reviews of sixteen drafts of eight sequences with the larger decoder vocabulary
        _logits("filter", "fp32", 136, 32128, "mixed", each=17, name="filter_batch"),
        # the logits of whole trees and blocks of many sequences, an odd vocabulary in half precision
        _logits("filter", "bf16", 656, 50001, "both", each=41, name="filter_trees_bf16"),
        # 64 sequences review four drafts each and keep none of them
        _pages(64, 16, 1, 4000, 5, name="pages_review"),
        # prompts enter while other sequences generate
        _pages(96, 16, 0, 9000, 4097, few=80, name="pages_prompts"),
        # the encoder-decoder shape reviews four drafts of one sequence against its encoder's 512 rows
        _cross("bf16", 1, 64, 1, 64, 16, 512, 512, 5, name="cross_review_bf16"),
        # a ragged batch of blocks over long e4m3 states, one of them empty
        _cross("fp8", 24, 8, 4, 128, 64, 0, 12000, 5, name="cross_batch_fp8"),
        # four decoder prompts over the encoder's states: the matrix cores bound this
        _cross("bf16", 4, 32, 1, 128, 64, 1000, 4096, 1024, name="cross_prompt_bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng: random.Random):
    kind = rng.choice(["sample", "sample", "filter", "filter", "pages", "cross", "cross"])
    if kind in ("sample", "filter"):
        vocab = rng.choice([512, 32000, 32128, _log(rng, 500, 131072), _log(rng, 500, 131072), _log(rng, 20000, 131072)])
        rows = _log(rng, 1, 656)
        most = 256 * 131072 if kind == "sample" else 656 * 50001
        each = rng.choice([1, 1, 5, 17])
        rows = max(1, min(rows, most // vocab) // each) * each
        return _logits(kind, rng.choice(["fp32", "fp32", "bf16"]), rows, vocab, rng.choice(["temperature", "top_k", "top_p", "min_p", "both", "mixed", "mixed"]),
                       pad=rng.choice([0, 0, 1, 37, 128]), each=each)
    if kind == "pages":
        batch, hi = _log(rng, 1, 512), _log(rng, 16, 9000)
        chunk = rng.choice([1, 5, 41, _log(rng, 1, 4097)])
        while batch * chunk > 16 * 4097 + 80:
            chunk = chunk * 3 // 4
        return _pages(batch, rng.choice([16, 32, 64, 128]), rng.randrange(0, hi + 1), hi, chunk, few=rng.randrange(batch) if rng.random() < 0.4 else 0)
    small = rng.random() < 0.15         # fp32: the small models
    cache = "fp32" if small else rng.choice(["bf16", "fp8"])
    d = rng.choice([16, 32, 64]) if small else rng.choice([64, 128])
    kv = rng.choice([2, 4]) if small else rng.choice([1, 4, 8, 12, 32, 64])
    group = rng.choice([1, 1, 4, 8]) if kv <= 8 else 1
    batch = _log(rng, 1, 4 if small else 64)
    chunk = _log(rng, 1, 32 if small else 1024)
    hi = _log(rng, 16, 1500 if small else 12000)
    few = rng.randrange(batch) if chunk > 1 and rng.random() < 0.3 else 0
    while batch * hi * kv * d > 2 ** 28 or batch * chunk * (hi + 1) * kv * group * d > 6e10 or batch * chunk * hi * kv * group > 5e8:
        if batch > 1 and rng.random() < 0.5:
            batch = max(1, batch * 3 // 4)
            few = min(few, batch - 1)
        elif hi > 64 and rng.random() < 0.5:
            hi = hi * 3 // 4
        else:
            chunk = max(1, chunk * 3 // 4)
    return _cross(cache, batch, kv, group, d, rng.choice([16, 32, 64, 128]), rng.randrange(0, hi + 1), hi, chunk, few=few, rows="fp32" if small else "bf16")


def _lengths(case):
    """(cached or encoded length, new rows) of each sequence: spread over lo .. hi, both of them present; the sequences with one new row come last."""
    n, lo, hi = case["batch"], case["lo"], case["hi"]
    cached = [hi if b == 0 else lo if b == 1 else lo + int((hi - lo) * (b * 0.6180339887 % 1.0)) for b in range(n)]
    new = [case["chunk"] if b < n - case["few"] else 1 for b in range(n)]
    return cached, new


def _quantise(x):
    """(codes, scale bytes) of rows [..., D] in fp32."""
    bits = x.abs().amax(-1).view(torch.int32)
    s = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(1, 254)
    inverse = ((254 - s) << 23).view(torch.float32)
    return (x * inverse[..., None]).to(torch.float8_e4m3fn), s.to(torch.uint8)


def _random_rows(shape, gen):
    """Rows as projections give them: a few features of every head are far larger than the rest."""
    x = torch.randn(shape, generator=gen, device="cuda")
    loud = torch.randint(0, shape[-1], (shape[-2], 2), generator=gen, device="cuda")
    gain = torch.ones(shape[-2:], device="cuda").scatter_(1, loud, 4.0)
    return x * gain


def _prepare_logits(c, gen, s):
    """Rows as language models give them: a wide bulk, and a number of likely tokens that differs from row to row."""
    wide = torch.empty((c.rows, c.vocab + c.pad), dtype=_TORCH[c.dtype], device="cuda")
    for at in range(0, c.rows, 64):
        n = min(64, c.rows - at)
        x = 2.0 * torch.randn((n, c.vocab + c.pad), generator=gen, device="cuda")
        likely = torch.randint(0, c.vocab, (n, 64), generator=gen, device="cuda")
        sharp = 5.0 + 7.0 * torch.rand((n, 1), generator=gen, device="cuda")
        x.scatter_(1, likely, sharp + 2.0 * torch.randn((n, 64), generator=gen, device="cuda"))
        wide[at:at + n] = x.to(wide.dtype)
    s.logits = wide[:, :c.vocab]
    s.u = torch.randint(0, 2 ** 24, (c.rows,), generator=gen, device="cuda").float() * 2.0 ** -24
    sets = c.rows // c.each
    rand = torch.rand((4, sets), generator=gen, device="cuda")
    s.temperature = 0.5 + 0.8 * rand[0]
    s.top_k = (1 + 99 * rand[1]).to(torch.int32) if c.by in ("top_k", "both", "mixed") else None
    s.top_p = 0.7 + 0.29 * rand[2] if c.by in ("top_p", "both", "mixed") else None
    s.min_p = 0.02 + 0.1 * rand[3] if c.by in ("min_p", "mixed") else None
    if c.by == "mixed":
        # sequences take what they want of it: which, by threes and fours; every eighth is greedy
        which = torch.arange(sets, device="cuda")
        s.top_k[which % 3 == 0] = 0
        s.top_p[which % 4 == 1] = 1.0
        s.min_p[which % 2 == 0] = 0.0
        s.temperature[which % 8 == 7] = 0.0


def _prepare_pages(c, gen, s):
    cached, new = _lengths(vars(c))
    held = [-(-t // c.page) for t in cached]
    whole = [-(-(t + m) // c.page) for t, m in zip(cached, new)]
    s.total = sum(new)
    n_pages = sum(whole) + 64
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    s.held = torch.tensor(held, dtype=torch.int32, device="cuda")
    at = torch.arange(max(whole) + 1, device="cuda")
    before = torch.cumsum(s.held, 0) - s.held
    s.table = torch.where(at < s.held[:, None], order[(before[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32)
    s.free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    s.free[:n_pages - sum(held)] = order[sum(held):]
    s.n_free = torch.tensor([n_pages - sum(held)], dtype=torch.int32, device="cuda")
    s.users = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    s.users[order[:sum(held)].long()] = 1
    s.cache_len = torch.tensor(cached, dtype=torch.int32, device="cuda")
    s.new_rows = torch.tensor(new, dtype=torch.int32, device="cuda")
    if own:
        import paper_2312_11462_amd as P
        s.pages = P.Pages(s.table, s.held, s.free, s.n_free, s.users, c.page)


def _prepare_cross(c, gen, s):
    length, new = _lengths(vars(c))
    pages = [-(-t // c.page) for t in length]
    n_pages = sum(pages) + 3
    s.max_rows, s.total, s.scale = max(new), sum(new), 1.0 if c.kv_heads == 64 else c.head_dim ** -0.5
    shape = (1, n_pages, c.kv_heads, c.page, c.head_dim)
    s.k = torch.empty(shape, dtype=_TORCH[c.cache], device="cuda")
    s.v = torch.empty_like(s.k)
    s.k_scale = s.v_scale = None
    if c.cache == "fp8":
        s.k_scale = torch.empty(shape[:-1], dtype=torch.uint8, device="cuda")
        s.v_scale = torch.empty_like(s.k_scale)
    for pool, scale in ((s.k, s.k_scale), (s.v, s.v_scale)):
        for at in range(0, n_pages, 4096):
            x = _random_rows((min(4096, n_pages - at), c.page, c.kv_heads, c.head_dim), gen).transpose(1, 2)
            if scale is None:
                pool[0, at:at + 4096] = x.to(pool.dtype)
            else:
                codes, scale[0, at:at + 4096] = _quantise(x)
                pool.view(torch.uint8)[0, at:at + 4096] = codes.view(torch.uint8)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    s.table = torch.zeros((c.batch, max(max(pages), 1)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        s.table[b, :n] = order[at:at + n]
        at += n
    s.enc_len = torch.tensor(length, dtype=torch.int32, device="cuda")
    s.row_start = torch.tensor([sum(new[:b]) for b in range(c.batch + 1)], dtype=torch.int32, device="cuda")
    # (unscaled attention has its factor in the query projection)
    s.q = (1.3 * c.head_dim ** -0.5 / s.scale * _random_rows((s.total, c.kv_heads * c.group, c.head_dim), gen)).to(_TORCH[c.rows])
    if own:
        import paper_2312_11462_amd as P
        s.kv = P.PagedKv(s.k, s.v, s.k_scale, s.v_scale)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c = SimpleNamespace(**case)
    s = SimpleNamespace(case=c)
    if c.kind == "pages":
        _prepare_pages(c, gen, s)
    elif c.kind == "cross":
        _prepare_cross(c, gen, s)
    else:
        _prepare_logits(c, gen, s)
    return s


def _weights(s):
    """Weights by token [rows][vocab] in 64 bits (sums that lie next to a border decide), 0 for the tokens that are left out."""
    c = s.case

    def of_row(t):
        return t.repeat_interleave(c.each)[:, None]
    top, order = torch.sort(s.logits, dim=-1, descending=True, stable=True)
    x = top.double()
    t = of_row(s.temperature).double()
    w = torch.exp((x - x[:, :1]) / torch.where(t > 0, t, 1.0))
    rank = torch.arange(c.vocab, device="cuda")
    keep = (t > 0) | (rank == 0)
    if s.top_k is not None:
        k = of_row(s.top_k)
        keep = keep & ((rank < k) | (k <= 0))
    w = w * keep
    if s.top_p is not None:
        p = of_row(s.top_p).double()
        run = torch.cumsum(w, -1)
        before = torch.nn.functional.pad(run[:, :-1], (1, 0))
        w = w * ((before < p * run[:, -1:]) | (p >= 1))
    if s.min_p is not None:
        w = w * (w >= of_row(s.min_p).double())
    return torch.zeros_like(w).scatter_(1, order, w)


def _plain_sample(s):
    run = torch.cumsum(_weights(s), -1)
    return torch.searchsorted(run, s.u.double()[:, None] * run[:, -1:], right=True)[:, 0].to(torch.int32)


def _plain_filter(s):
    w = _weights(s)
    return (w / w.sum(-1, keepdim=True)).float()


def _plain_pages(s):
    c = s.case
    room = s.table.shape[1]
    at = torch.arange(room, device="cuda")
    # the step's rows enter
    wanted = (s.cache_len + s.new_rows + c.page - 1) // c.page
    fits = wanted <= room
    need, rows = (wanted - s.held).clamp(min=0) * fits, s.new_rows * fits
    served = fits & ((need == 0) | (torch.cumsum(need, 0) <= s.n_free)) & ((rows == 0) | (torch.cumsum(rows, 0) <= s.total))
    need, rows = need * served, rows * served
    rank = torch.cumsum(need, 0) - need
    fresh = (at >= s.held[:, None]) & (at < (s.held + need)[:, None])
    take = s.n_free - 1 - (rank[:, None] + at - s.held[:, None])
    s.table.copy_(torch.where(fresh, s.free[take.clamp(0, s.free.numel() - 1)], s.table))
    s.users.index_add_(0, s.table.clamp(min=0).view(-1), fresh.view(-1).int())
    s.held.add_(need)
    s.n_free.sub_(need.sum())
    row_start = torch.nn.functional.pad(torch.cumsum(rows, 0), (1, 0)).to(torch.int32)
    r = torch.arange(s.total, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(row_start, r, right=True) - 1
    there = b < c.batch
    b = b.clamp(max=c.batch - 1)
    pos = s.cache_len[b] + r - row_start[b]
    slot = s.table[b, pos // c.page].long() * c.page + pos % c.page
    out = [row_start, torch.where(there, b, -1).to(torch.int32), torch.where(there, pos, -1).to(torch.int32), torch.where(there, slot, -1), served.to(torch.int32)]
    # and are not kept: pages behind the cached rows go back, so that they are taken in the same order again
    kept = torch.minimum((s.cache_len + c.page - 1) // c.page, s.held)
    gone = (at >= kept[:, None]) & (at < s.held[:, None])
    page = s.table.clamp(min=0)
    s.users.index_add_(0, page.view(-1), -gone.view(-1).int())
    index = torch.arange(gone.numel(), device="cuda").view_as(gone)
    empty = gone & (s.users[page] == 0)
    first = torch.full((s.users.numel() + 1,), gone.numel(), device="cuda").scatter_reduce_(0, torch.where(empty, page, s.users.numel()).view(-1).long(),
                                                                                               index.view(-1), "amin")
    back = (empty & (first[page] == index)).view(-1)
    rank = torch.cumsum(back, 0) - 1
    n = back.sum()
    longer = torch.nn.functional.pad(s.free, (0, 1))
    longer.scatter_(0, torch.where(back, s.n_free + n - 1 - rank, s.free.numel()), page.view(-1))
    s.free.copy_(longer[:-1])
    s.n_free.add_(n)
    s.table.masked_fill_(gone, -1)
    s.held.copy_(kept)
    return out + [s.table, s.held, s.free, s.n_free, s.users]


def _plain_cross(s):
    c = s.case
    n, m, g, d = c.batch, s.max_rows, c.group, c.head_dim
    keys = s.table.shape[1] * c.page
    at = torch.arange(keys, device="cuda")
    page, slot = s.table[:, at // c.page].long(), (at % c.page)[None]

    def rows_of(pool, scale):
        x = pool.view(torch.uint8)[0][page, :, slot].view(pool.dtype) if scale is not None else pool[0][page, :, slot]
        x = x.float()
        return x if scale is None else x * (scale[0][page, :, slot].int() << 23).view(torch.float32)[..., None]
    inside = at[None] < s.enc_len[:, None]
    k = rows_of(s.k, s.k_scale).permute(0, 2, 3, 1).contiguous()      # [n][kv][D][keys]
    v = rows_of(s.v, s.v_scale).permute(0, 2, 1, 3).contiguous()      # [n][kv][keys][D]
    i = torch.arange(m, device="cuda")
    row = torch.minimum(s.row_start[:-1, None] + i[None], s.row_start[1:, None] - 1)
    q = s.q[row].float().view(n, m, c.kv_heads, g, d).permute(0, 2, 3, 1, 4).reshape(n, c.kv_heads, g * m, d)
    scores = torch.matmul(q.contiguous(), k).mul_(s.scale).masked_fill_(~inside[:, None, None], float("-inf"))
    p = scores.sub_(scores.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    p.div_(p.sum(-1, keepdim=True).clamp(min=1e-30))
    o = torch.matmul(p, v).view(n, c.kv_heads, g, m, d).permute(0, 3, 1, 2, 4)
    r = torch.arange(s.total, device="cuda")
    b = torch.searchsorted(s.row_start, r.to(torch.int32), right=True) - 1
    return o[b, r - s.row_start[b]].reshape(s.total, c.kv_heads * g, d).to(s.q.dtype)


def run(s):
    c = s.case
    if c.kind == "cross":
        return s.kv.cross_attention(0, s.table, s.row_start, s.enc_len, s.q, s.scale, s.max_rows) if own else _plain_cross(s)
    if c.kind == "pages":
        if not own:
            return _plain_pages(s)
        out = s.pages.plan(s.cache_len, s.new_rows, s.total)
        s.pages.release(s.cache_len)
        return [*out, s.table, s.held, s.free, s.n_free, s.users]
    if not own:
        return _plain_sample(s) if c.kind == "sample" else _plain_filter(s)
    import paper_2312_11462_amd as P
    settings = dict(temperature=s.temperature, top_k=s.top_k, top_p=s.top_p, min_p=s.min_p)
    return P.sample(s.logits, s.u, **settings) if c.kind == "sample" else P.filter_probs(s.logits, **settings)


def work(case):
    c = SimpleNamespace(**case)
    if c.kind in ("sample", "filter"):
        # an exponential, its sum and the draw's running sum at least
        return {"bytes": c.rows * c.vocab * (_SIZE[c.dtype] + (4 if c.kind == "filter" else 0)) + 4 * c.rows, "flops": 3 * c.rows * c.vocab}
    cached, new = _lengths(case)
    if c.kind == "pages":
        # lengths, pages held and the row starts, twice; sequence, position and slot of a row; table, users and stack of a page, taken and given back
        taken = sum(-(-(t + m) // c.page) - -(-t // c.page) for t, m in zip(cached, new))
        return {"bytes": 32 * c.batch + 16 * sum(new) + 36 * taken, "flops": 0}
    per_row = c.kv_heads * (c.head_dim * _SIZE[c.cache] + (1 if c.cache == "fp8" else 0)) * 2     # K and V of an encoder's row
    heads = c.kv_heads * c.group
    return {"bytes": sum(cached) * per_row + sum(new) * heads * c.head_dim * _SIZE[c.rows] * 2,
            "flops": 4 * sum(m * t for t, m in zip(cached, new)) * heads * c.head_dim}


def exact(case, seed):
    s = prepare(case, seed)
    c = s.case
    if c.kind in ("sample", "pages"):
        return None                     # whole numbers
    if c.kind == "filter":
        out = torch.zeros((c.rows, c.vocab), dtype=torch.float64, device="cuda")
        index = torch.arange(c.vocab, device="cuda")
        sets = [[1.0 if v is None else float(v[i]) for v in (s.temperature, s.top_p)] + [0 if s.top_k is None else int(s.top_k[i])]
                + [0.0 if s.min_p is None else float(s.min_p[i])] for i in range(c.rows // c.each)]
        for r in range(c.rows):
            t, p, k, least = sets[r // c.each]
            x = s.logits[r].to(torch.float64)
            best = int(torch.min(index[x == x.max()]))
            if t <= 0:
                out[r, best] = 1
                continue
            weight = torch.exp(x / t - x[best] / t)
            # a rank for each token: by a sort of the negated logits that keeps equal ones in their order
            by = torch.argsort(-x, stable=True)
            if 0 < k < c.vocab:
                by = by[:k]
            mass = weight[by]
            if p < 1:
                total = mass.sum()
                behind = total - torch.cumsum(mass, 0)                # what is left behind each of them
                n = int((behind > (1 - p) * total).sum()) + 1
                by = by[:n]
            by = by[weight[by] >= least]
            out[r, by] = weight[by] / weight[by].sum()
        return out
    out, at = [], 0
    length, new = _lengths(case)
    for b, (t, m) in enumerate(zip(length, new)):
        q = s.q[at:at + m].to(torch.float64)
        at += m
        if t == 0:
            out.append(torch.zeros_like(q))
            continue
        pos = torch.arange(t, device="cuda")
        page, slot = s.table[b].long()[torch.div(pos, c.page, rounding_mode="floor")], torch.remainder(pos, c.page)
        side = []
        for pool, scale in ((s.k, s.k_scale), (s.v, s.v_scale)):
            x = pool[0].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn) if scale is not None else pool[0][page, :, slot]
            x = x.to(torch.float64)
            side.append(x if scale is None else x * torch.pow(2.0, scale[0][page, :, slot].to(torch.float64) - 127)[..., None])
        heads = [torch.softmax((q[:, h] @ side[0][:, h // c.group].t().contiguous()) * s.scale, dim=-1) @ side[1][:, h // c.group].contiguous()
                 for h in range(c.kv_heads * c.group)]
        out.append(torch.stack(heads, 1))
    return torch.cat(out)
