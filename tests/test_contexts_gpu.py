"""Attention over shared and sparse contexts of the paged cache: a shared beginning read once, summaries of pages, the choice of pages, the attention over the chosen ones; against plain
implementations in 64 bits (numpy), whole numbers to the bit."""
import numpy as np
import pytest

from test_paged_gpu import HEADS, Batch, attention64, check, f16, filled, held

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P(_built_library):
    import paper_2505_00232_b200 as P
    return P


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    return torch


def dev(torch, a):
    return torch.tensor(np.array(a, dtype=np.int32, order="C"), dtype=torch.int32, device="cuda")


def bounds64(k):
    """(largest, smallest, unit) of a page's keys [tokens, h_kv, d], fp16 values: fp32 operations, each rounded once."""
    k = k.astype(np.float16).astype(np.float32)
    hi, lo = k.max(0), k.min(0)
    top = np.maximum(hi, -lo).max(-1)
    with np.errstate(divide="ignore"):
        r = np.where(top > 0, np.float32(127) / top, np.float32(0))[:, None].astype(np.float32)
    return np.minimum(np.ceil(hi * r), 127), np.maximum(np.floor(lo * r), -127), (top / np.float32(127)).astype(np.float32)


def chosen64(q, h_kv, bounds, scales, row, pos, page, n_pages, budget, first, recent):
    """The columns chosen for a row's queries [h_q, d]: [h_kv, budget]."""
    h_q, d = q.shape
    last = min(pos // page, len(row) - 1) if pos >= 0 else -1
    ok = np.array([0 <= x < n_pages for x in row[:last + 1]], bool)
    out = np.full((h_kv, budget), -1)
    for h in range(h_kv):
        up, down = np.zeros(d, np.float32), np.zeros(d, np.float32)
        for x in q[h * (h_q // h_kv):(h + 1) * (h_q // h_kv)].astype(np.float32):
            up, down = up + np.maximum(x, 0), down + np.minimum(x, 0)
        top = max(up.max(), -down.min())
        r = np.float32(32767) / top if top > 0 else np.float32(0)
        up, down = (np.rint(v * r).astype(np.int64) for v in (up, down))
        at = np.where(ok, row[:last + 1], 0)
        total = bounds[at, h, 0].astype(np.int64) @ up + bounds[at, h, 1].astype(np.int64) @ down
        score = total.astype(np.float32) * scales[at, h]
        c = np.arange(last + 1)
        always = (c < first) | (c > last - recent)
        order = sorted(np.flatnonzero(ok).tolist(), key=lambda j: (not always[j], 0.0 if always[j] else -score[j], j))[:budget]
        out[h, :len(order)] = sorted(order)
    return out


def attended64(q, k, v, scale, softcap=0.0):
    """(out, bound) of one KV head's queries [g, d] over the tokens k, v [n, d], in 64 bits: the roundings that attention64 counts, without those of the keys."""
    g, d = q.shape
    if len(k) == 0:
        return np.zeros((g, d)), np.zeros((g, d))
    q64 = q.astype(np.float64)
    x = q64 @ k.T * scale
    dx = (d + 40) * 2.0 ** -24 * (np.abs(q64) @ np.abs(k).T) * abs(scale)
    if softcap:
        x = softcap * np.tanh(x / softcap)
        dx = dx + 16 * 2.0 ** -24 * softcap
    w = np.exp(x - x.max(-1, keepdims=True))
    p = w / w.sum(-1, keepdims=True)
    rel = np.expm1(dx + 2.0 ** -21 * (1 + np.abs(x - x.max(-1, keepdims=True)))).max(-1, keepdims=True)
    y, a = p @ v, p @ np.abs(v)
    e = (2 * rel + 2 * 2.0 ** -11 + len(k) * 2.0 ** -24) * a + 2.0 ** -25 / w.sum(-1, keepdims=True) * np.abs(v).sum(0)
    return y, 1.01 * e + 2.0 ** -11 * np.abs(y) + 2.0 ** -25


# ---------------------------------------------------------------------------- summaries
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_summaries(P, torch, h_q, h_kv, d, page):
    """Of the pages that new tokens lie in, over the tokens so far; the others stay."""
    lens, new = [1, 37, 16, 700, 5, 256, 300], [1, 5, 16, 300, 0, 1, 45]
    batch = Batch(torch, lens, new, page, seed=page + d, before=3, behind=2)
    cache, kv = filled(P, torch, batch, h_kv, d)
    bounds, scales = cache.key_bounds()
    bounds.fill_(99)
    scales.fill_(7.5)
    cache.summarise((bounds, scales), *batch.args, batch.T)
    want, want_s = np.full(bounds.shape, 99), np.full(scales.shape, 7.5, np.float32)
    for b, (n, m) in enumerate(zip(lens, batch.new)):
        for j in range((n - m) // page, (n - 1) // page + 1) if m else ():
            x = batch.table[b, j]
            want[x, :, 0], want[x, :, 1], want_s[x] = bounds64(kv[b][0][j * page:min(n, (j + 1) * page)])
    assert (bounds.cpu().numpy() == want).all() and (scales.cpu().numpy() == want_s).all()


def test_summaries_token_by_token_equal_those_at_once(P, torch):
    rng = np.random.default_rng(2)
    n, page, h_kv, d = 77, 32, 2, 128
    batch = Batch(torch, [n], [n], page)
    k, v = (torch.from_numpy(f16(rng, n, h_kv, d)).cuda() for _ in range(2))
    cache = P.PagedKV(batch.n_pages, page, h_kv, d)
    once, steps = cache.key_bounds(), cache.key_bounds()
    for i in range(n):
        at = (batch.args[0], dev(torch, [i + 1]), dev(torch, [0, 1]))
        cache.append(k[i:i + 1], v[i:i + 1], *at)
        cache.summarise(steps, *at, 1)
    cache.summarise(once, *batch.args, n)
    assert torch.equal(once[0], steps[0]) and torch.equal(once[1], steps[1])


def test_summaries_at_the_edge(P, torch):
    """Zero keys, entries without a page, lengths and rows that are none, a length beyond the table."""
    page, h_kv, d = 16, 1, 64
    cache = P.PagedKV(20, page, h_kv, d)
    b = cache.key_bounds()
    b[0].fill_(5)
    table = np.full((6, 3), -1)
    table[0], table[1, 0], table[2], table[3], table[4] = [3, 20, 4], 5, [6, 7, 8], [9, 10, 11], [12, 13, 14]
    cache.summarise(b, dev(torch, table), dev(torch, [40, 0, -9, 2 ** 31 - 1, 5, 10]), dev(torch, [0, 40, 42, 44, 50, 58, 90]), 60)
    touched = {3, 4, 12}                                                 # (sequence 3's new rows lie beyond the table, sequence 5's are not in the call)
    got = b[0].cpu().numpy()
    assert all((got[x] == (0 if x in touched else 5)).all() for x in range(20)) and (b[1] == 0).all()
    cache.summarise(b, dev(torch, table)[:0], dev(torch, []), dev(torch, [0]), 0)


# ---------------------------------------------------------------------------- the choice of pages
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("page,budget,first,recent", [(16, 5, 1, 1), (16, 1, 0, 0), (32, 40, 0, 3), (64, 3, 3, 0), (16, 129, 2, 2)])
def test_select(P, torch, h_q, h_kv, d, page, budget, first, recent):
    rng = np.random.default_rng(page + budget)
    lens, new = [1, 37, 16, 2100, 5, 900, 1500], [1, 2, 16, 3, 0, 1, 1]
    batch = Batch(torch, lens, new, page, seed=page + d, before=3, behind=2)
    batch.table[5, 2], batch.table[5, 1] = -1, batch.n_pages              # (columns without a page)
    args = (dev(torch, batch.table), *batch.args[1:])
    cache = P.PagedKV(batch.n_pages, page, h_kv, d)
    shape = (batch.n_pages, h_kv, 2, d)
    bounds = np.sort(rng.integers(-127, 128, shape), 2)[:, :, ::-1].astype(np.int8)
    scales = rng.random(shape[:2]).astype(np.float32) + np.float32(0.1)
    bounds[: batch.n_pages // 2] = bounds[0]                             # (half of the pages are the same: ties)
    scales[: batch.n_pages // 2] = scales[0]
    q = f16(rng, batch.T, h_q, d)
    q[4] = 0                                                             # (all the same)
    out = torch.full((batch.T, h_kv, budget), 77, dtype=torch.int32, device="cuda")
    dq = torch.from_numpy(q).cuda()
    db = torch.from_numpy(bounds.copy()).cuda(), torch.from_numpy(scales).cuda()
    assert cache.select(dq, db, *args, budget, first, recent, out=out) is out
    want = np.full(out.shape, 77)
    for t, b, pos in batch.rows():
        want[t] = chosen64(q[t], h_kv, bounds, scales, batch.table[b], pos, page, batch.n_pages, budget, first, recent)
    assert (out.cpu().numpy() == want).all()
    wide = torch.zeros((batch.T, h_q * d + 64), dtype=torch.float16, device="cuda")   # (rows of a wider projection; the Python half, another stream)
    wide[:, :h_q * d] = dq.view(batch.T, -1)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    again = cache.select(wide[:, :h_q * d], db, *args, budget, first, recent, stream=stream)
    stream.synchronize()
    rows = [r[0] for r in batch.rows()]
    assert (again.cpu().numpy()[rows] == want[rows]).all()


@pytest.mark.parametrize("W,B,budget", [(260, 1, 64), (1100, 3, 32), (9000, 1, 700), (70001, 2, 50), (262144, 1, 3)])
def test_select_from_many_pages(P, torch, W, B, budget):
    """Wide tables, by clusters; a few thousand different summaries, so that ties are many."""
    rng = np.random.default_rng(W)
    h_q, h_kv, d, page, n_pages = 4, 2, 64, 16, 5000
    cache = P.PagedKV(n_pages, page, h_kv, d)
    bounds = np.sort(rng.integers(-127, 128, (n_pages, h_kv, 2, d)), 2)[:, :, ::-1].astype(np.int8)
    scales = rng.random((n_pages, h_kv)).astype(np.float32)
    table = rng.integers(-1, n_pages, (B, W))
    lens = [W * page - 3] + [W * page // (2 + b) for b in range(B - 1)]
    q = f16(rng, B, h_q, d)
    got = cache.select(torch.from_numpy(q).cuda(), (torch.from_numpy(bounds.copy()).cuda(), torch.from_numpy(scales).cuda()), dev(torch, table), dev(torch, lens), dev(torch, range(B + 1)), budget).cpu().numpy()
    for b in range(B):
        assert (got[b] == chosen64(q[b], h_kv, bounds, scales, table[b], lens[b] - 1, page, n_pages, budget, 1, 1)).all()


def test_select_for_many_rows(P, torch):
    """A prompt's rows, each with its own choice."""
    rng = np.random.default_rng(9)
    h_q, h_kv, d, page, n = 4, 2, 128, 16, 700
    batch = Batch(torch, [n, 40], [n, 40], page)
    cache, kv = filled(P, torch, batch, h_kv, d)
    b = cache.key_bounds()
    cache.summarise(b, *batch.args, batch.T)
    q = f16(rng, batch.T, h_q, d)
    got = cache.select(torch.from_numpy(q).cuda(), b, *batch.args, 6, 1, 2).cpu().numpy()
    bounds, scales = (x.cpu().numpy() for x in b)
    for t, s, pos in batch.rows()[::7]:
        assert (got[t] == chosen64(q[t], h_kv, bounds, scales, batch.table[s], pos, page, batch.n_pages, 6, 1, 2)).all()


def test_a_bound_is_one(P, torch):
    """No token's score, summed over a KV head's queries, passes its page's but by the codes' rounding."""
    rng = np.random.default_rng(4)
    h_q, h_kv, d, page, n = 8, 2, 128, 32, 600
    batch = Batch(torch, [n], [1], page)
    cache, kv = filled(P, torch, batch, h_kv, d)
    b = cache.key_bounds()
    cache.summarise(b, *batch.whole, n)
    bounds, scales = (x.cpu().numpy().astype(np.float64) for x in b)
    q = f16(rng, h_q, d).astype(np.float64)
    for h in range(h_kv):
        g = q[4 * h:4 * h + 4]
        for j in range(-(-n // page)):
            x = batch.table[0, j]
            hi, lo = (bounds[x, h, i] * scales[x, h] for i in range(2))
            bound = np.maximum(g, 0).sum(0) @ hi + np.minimum(g, 0).sum(0) @ lo
            scores = (kv[0][0][j * page:(j + 1) * page, h] @ g.T).sum(-1)
            slack = 2.0 ** -11 * (np.abs(kv[0][0][j * page:(j + 1) * page, h]) @ np.abs(g).T).sum(-1).max()   # (the bounds are of fp16(q s); the products of their fp32 operations)
            assert scores.max() <= bound + slack


# ---------------------------------------------------------------------------- attention over listed pages
@pytest.mark.parametrize("h_q,h_kv,d", HEADS + [(64, 2, 64)])
@pytest.mark.parametrize("page,budget,scale,softcap", [(16, 9, 1.0, 0.0), (64, 4, -0.7, 0.0), (32, 30, 1.0, 20.0), (128, 2, 1.0, 500.0), (16, 1, 1.0, 0.0)])
def test_attention_selected(P, torch, h_q, h_kv, d, page, budget, scale, softcap):
    """Lists in any order, the same column twice, columns that are none, without a page or behind the row; rows of no sequence stay."""
    rng = np.random.default_rng(page + budget + d)
    lens, new = [1, 37, 16, 1300, 5, 900], [1, 2, 16, 3, 0, 1]
    batch = Batch(torch, lens, new, page, seed=page + d, before=3, behind=2)
    cache, kv = filled(P, torch, batch, h_kv, d)
    W = batch.table.shape[1]
    batch.table[5, 1] = -1
    args = (dev(torch, batch.table), *batch.args[1:])
    pages = rng.integers(-1, W + 1, (batch.T, h_kv, budget))
    pages[:, 0] = np.sort(pages[:, 0])                                   # (one head's in order)
    pages[4] = -1
    pages[-3, 0, 0], pages[-3, -1, 0] = 2 ** 31 - 1, -2 ** 31
    q, scale = f16(rng, batch.T, h_q, d), scale / np.sqrt(d)
    out = torch.full((batch.T, h_q, d), 7.5, dtype=torch.float16, device="cuda")
    assert cache.attention_selected(torch.from_numpy(q).cuda(), dev(torch, pages), *args, scale=scale, softcap=softcap, out=out) is out
    got, g = out.cpu().numpy().astype(np.float64), h_q // h_kv
    rows = batch.rows()
    for t, b, pos in rows:
        for h in range(h_kv):
            tokens = [j for c in pages[t, h, :min(budget, -(-lens[b] // page))] if 0 <= c < W and 0 <= batch.table[b, c] < batch.n_pages for j in range(c * page, min((c + 1) * page, pos + 1))]
            y, tol = attended64(q[t, g * h:g * h + g], kv[b][0][tokens, h], kv[b][1][tokens, h], scale, softcap)
            assert (np.abs(got[t, g * h:g * h + g] - y) <= tol).all(), (t, h)
    rest = np.setdiff1d(np.arange(batch.T), [r[0] for r in rows])
    assert (got[rest] == 7.5).all()


@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("B", [1, 3, 70])
def test_attention_over_every_page_is_attention(P, torch, h_q, h_kv, d, B):
    """Long lists that CTAs share, batches of many segments: the definition over whole sequences."""
    rng = np.random.default_rng(B + d)
    lens = [5000 // min(B, 4)] + [int(n) for n in rng.integers(1, 5000 // B + 2, B - 1)]
    batch = Batch(torch, lens, [1 + b % 3 for b in range(B)], 32, seed=B)
    cache, kv = filled(P, torch, batch, h_kv, d)
    W = batch.table.shape[1]
    pages = np.broadcast_to(np.arange(W), (batch.T, h_kv, W))
    q = f16(rng, batch.T, h_q, d)
    run = lambda: cache.attention_selected(torch.from_numpy(q).cuda(), dev(torch, pages), *batch.args)
    got = run()
    want, tol = attention64(q, kv, batch, d ** -0.5, max_q=1)
    check(got.cpu().numpy(), want, tol, batch.rows())
    for _ in range(5):
        assert torch.equal(run(), got)


def test_rows_before_the_first_token_and_empty_lists(P, torch):
    cache = P.PagedKV(8, 16, 1, 64)
    q = torch.randn(12, 2, 64, device="cuda").half()
    table, kv, start = dev(torch, [[0, 1], [2, 3], [4, 5]]), dev(torch, [3, 0, -7]), dev(torch, [0, 6, 9, 12])
    b = cache.key_bounds()
    got = cache.select(q, b, table, kv, start, 2, 0, 0).cpu().numpy()
    assert (got[:3] == -1).all() and (got[3:6] == [0, -1]).all() and (got[6:] == -1).all()
    out = torch.full_like(q, 7.5)
    cache.attention_selected(q, dev(torch, np.zeros((12, 1, 2))), table, kv, start, out=out)
    assert (out[:3] == 0).all() and (out[6:] == 0).all()                 # (and the cache holds zeros: so are the others)
    out.fill_(7.5)
    cache.attention_selected(q, torch.empty((12, 1, 0), dtype=torch.int32, device="cuda"), table, kv, start, out=out)
    assert (out == 0).all()


# ---------------------------------------------------------------------------- a shared beginning
def sharing(P, torch, groups, page, h_kv, d, new, seed=0, before=0, behind=0, alone=()):
    """groups: (prefix, own lengths); their sequences in order, those of `alone` behind them.  Whole pages of a prefix are the same pages, what is left of it is held twice.
    (cache, batch, its keys and values, group_start, prefix_len)"""
    lens = [n + p for p, own in groups for n in own] + list(alone)
    batch = Batch(torch, lens, [new] * len(lens) if np.isscalar(new) else new, page, seed, before, behind)
    cache, kv = filled(P, torch, batch, h_kv, d, seed + 1)
    b, start = 0, [0]
    rng = np.random.default_rng(seed + 2)
    k, v = (f16(rng, sum(lens), h_kv, d) for _ in range(2))
    ends = np.cumsum(lens)
    for p, own in groups:
        first = ends[b] - lens[b]
        for i in range(b, b + len(own)):
            at = ends[i] - lens[i]
            k[at:at + p], v[at:at + p] = k[first:first + p], v[first:first + p]
            batch.table[i, :p // page] = batch.table[b, :p // page]
        b += len(own)
        start.append(b)
    args = dev(torch, batch.table)
    batch.args, batch.whole = (args, *batch.args[1:]), (args, *batch.whole[1:])
    for i in range(len(lens)):                                           # (one sequence after the other: they write the same bytes to a shared page)
        at = slice(ends[i] - lens[i], ends[i])
        cache.append(torch.from_numpy(k[at]).cuda(), torch.from_numpy(v[at]).cuda(), args[i:i + 1], batch.args[1][i:i + 1], dev(torch, [0, lens[i]]))
    kv = [(held(k[e - n:e]), held(v[e - n:e])) for e, n in zip(ends, lens)]
    return cache, batch, kv, dev(torch, start), dev(torch, [p for p, _ in groups])


GROUPS = [([(64, [1, 2])], 1, 0.0), ([(200, [30, 1, 77])], 1, 0.0), ([(1000, [5] * 20), (130, [100, 9]), (63, [8, 300])], 1, 0.0), ([(700, [40, 50, 60, 70, 80])], 5, 30.0), ([(3000, [50] * 40)], 1, 0.0),
          ([(512, [600, 20, 90]), (1024, [9] * 9)], 9, 0.0), ([(320, [64] * 70)], 2, 0.0), ([(100, [1])], 1, 0.0), ([(2048, [400, 300])], 40, 0.0)]


@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("groups,new,softcap", GROUPS)
def test_attention_shared(P, torch, h_q, h_kv, d, groups, new, softcap):
    """(max_q of attention64: the keys' rounding, which the kernel of many rows makes, counts whichever kernel takes a stretch.)"""
    rng = np.random.default_rng(d + len(groups))
    cache, batch, kv, start, prefix = sharing(P, torch, groups, 32, h_kv, d, new, seed=d, before=2, behind=3, alone=[17, 400])
    q = f16(rng, batch.T, h_q, d)
    out = torch.full((batch.T, h_q, d), 7.5, dtype=torch.float16, device="cuda")
    dq = torch.from_numpy(q).cuda()
    assert cache.attention_shared(dq, *batch.args, batch.max_q, start, prefix, softcap=softcap, out=out) is out
    want, tol = attention64(q, kv, batch, d ** -0.5, softcap, max_q=10 ** 6)
    check(out.cpu().numpy(), want, tol, batch.rows())
    rest = np.setdiff1d(np.arange(batch.T), [r[0] for r in batch.rows()])
    assert (out.cpu().numpy()[rest] == 7.5).all()
    again = torch.full_like(out, 7.5)
    for _ in range(4):
        cache.attention_shared(dq, *batch.args, batch.max_q, start, prefix, softcap=softcap, out=again)
        assert torch.equal(again, out)


@pytest.mark.parametrize("h_q,h_kv,d", [(32, 8, 128), (8, 4, 256), (14, 2, 64)])
def test_prefixes_that_not_all_rows_see(P, torch, h_q, h_kv, d):
    """A prefix longer than a sequence, rows inside it, no rows, groups that are none, rows beyond max_q, negative scales."""
    rng = np.random.default_rng(d)
    groups = [(640, [0, 100, 40]), (300, [20, 30]), (256, [200, 100])]
    new = [3, 700, 0, 2, 2, 9, 2, 1]
    cache, batch, kv, start, prefix = sharing(P, torch, groups, 16, h_kv, d, new, seed=3, alone=[50])
    q, scale = f16(rng, batch.T, h_q, d), -1.3 * d ** -0.5
    dq = torch.from_numpy(q).cuda()
    want, tol = attention64(q, kv, batch, scale, max_q=10 ** 6)
    starts = [start.tolist(), [0, 3, 3, 5], [-1, 3, 5, 7], [0, 3, 5, 99], [5, 3, 0, 0], [2, 3, 5, 7], [0, 0, 0, 8]]
    for s in starts:
        lens = prefix.tolist() if s == starts[0] else [2 ** 31 - 1, 300, -5] if s[0] < 0 else [0, 300, 250]
        if s == starts[-1]:
            lens = [0, 0, 0]
        for max_q in (4, 9):
            out = torch.full((batch.T, h_q, d), 7.5, dtype=torch.float16, device="cuda")
            cache.attention_shared(dq, *batch.args, max_q, dev(torch, s), dev(torch, lens), scale=scale, out=out)
            rows = [(t, b, pos) for t, b, pos in batch.rows() if t - batch.starts[b] < max_q]
            check(out.cpu().numpy(), want, tol, rows)
            rest = np.setdiff1d(np.arange(batch.T), [r[0] for r in rows])
            assert (out.cpu().numpy()[rest] == 7.5).all()


def test_prompts_behind_a_shared_prefix(P, torch):
    """Sequences whose own rows fill a tile read what they see once already: the call is attention's, to the bit."""
    rng = np.random.default_rng(1)
    cache, batch, kv, start, prefix = sharing(P, torch, [(500, [300, 200])], 16, 2, 128, [300, 200], seed=5)
    q = torch.from_numpy(f16(rng, batch.T, 8, 128)).cuda()
    assert torch.equal(cache.attention_shared(q, *batch.args, 300, start, prefix), cache.attention(q, *batch.args, 300))
    assert torch.equal(cache.attention_shared(q, *batch.args, 300, start[:1], prefix[:0]), cache.attention(q, *batch.args, 300))


def test_nothing_seen_and_nothing_to_do(P, torch):
    cache = P.PagedKV(8, 16, 1, 64)
    q = torch.randn(9, 2, 64, device="cuda").half()
    table, kv, start = dev(torch, [[-1, -1], [-1, 9], [0, 1]]), dev(torch, [20, 30, 0]), dev(torch, [0, 3, 6, 9])
    out = torch.full_like(q, 7.5)
    cache.attention_shared(q, table, kv, start, 3, dev(torch, [0, 3]), dev(torch, [16]), out=out)
    assert (out == 0).all()
    assert cache.attention_shared(q[:0], table[:0], kv[:0], start[:1], 3, dev(torch, [0, 0]), dev(torch, [5])).shape == (0, 2, 64)
    none = dev(torch, [])
    assert cache.select(q[:0], cache.key_bounds(), table[:0], none, start[:1], 3).shape == (0, 1, 3)
    assert cache.attention_selected(q[:0], torch.empty((0, 1, 3), dtype=torch.int32, device="cuda"), table[:0], none, start[:1]).shape == (0, 2, 64)


def test_long_shared_prefix(P, torch):
    """More steps than a CTA's share, many row tiles: 200 sequences over 6000 tokens, in tiles and, with few rows a group, not."""
    rng = np.random.default_rng(8)
    for groups, h_q, h_kv in (([(6000, [3] * 200)], 8, 2), ([(6000, [70, 2])], 4, 2), ([(6000, [70, 2, 9])] * 4, 4, 2)):
        cache, batch, kv, start, prefix = sharing(P, torch, groups, 64, h_kv, 128, 1, seed=4)
        q = f16(rng, batch.T, h_q, 128)
        got = cache.attention_shared(torch.from_numpy(q).cuda(), *batch.args, 1, start, prefix)
        want, tol = attention64(q, kv, batch, 128 ** -0.5, max_q=10 ** 6)
        check(got.cpu().numpy(), want, tol, batch.rows())


# ---------------------------------------------------------------------------- all of it, as a serving loop uses it
def test_requests_that_share_a_prompt(P, torch):
    """A prompt is cached once, forked for three continuations, each step reserves, appends, summarises, attends over all and over chosen pages; one ends, the pool is compacted, the others go on.  Every attention is
    checked against the tokens that the continuations really have; the steps are one captured graph."""
    rng = np.random.default_rng(11)
    h_q, h_kv, d, page, n_pages, W = 8, 2, 128, 16, 90, 24
    cache = P.PagedKV(n_pages, page, h_kv, d)
    bounds = cache.key_bounds()
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    prompt = 133
    root = torch.full((1, W), -1, dtype=torch.int32, device="cuda")
    at = root, dev(torch, [prompt]), dev(torch, [0, prompt])
    k0, v0 = f16(rng, prompt, h_kv, d), f16(rng, prompt, h_kv, d)
    assert cache.reserve(refs, *at, prompt).tolist() == [0]
    cache.append(torch.from_numpy(k0).cuda(), torch.from_numpy(v0).cuda(), *at)
    cache.summarise(bounds, *at, prompt)
    n = 3
    table = cache.fork(refs, root, dev(torch, [0] * n), dev(torch, [prompt] * n))
    cache.release(refs, root, dev(torch, [0]))
    kv_len, start = dev(torch, [prompt] * n), dev(torch, range(n + 1))
    group, prefix = dev(torch, [0, n]), dev(torch, [prompt])
    q = torch.zeros((n, h_q, d), dtype=torch.float16, device="cuda")
    k, v = (torch.zeros((n, h_kv, d), dtype=torch.float16, device="cuda") for _ in range(2))

    def step():
        kv_len.add_(1)
        missing = cache.reserve(refs, table, kv_len, start, n)
        cache.append(k, v, table, kv_len, start)
        cache.summarise(bounds, table, kv_len, start, n)
        whole = cache.attention_shared(q, table, kv_len, start, 1, group, prefix)
        pages = cache.select(q, bounds, table, kv_len, start, 5, 1, 2)
        return missing, whole, pages, cache.attention_selected(q, pages, table, kv_len, start)

    keep = [x.clone() for x in (kv_len, refs, table, cache.pool, *bounds)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step()
    for x, y in zip((kv_len, refs, table, cache.pool, *bounds), keep):
        x.copy_(y)
    ks, vs = [[k0] for _ in range(n)], [[v0] for _ in range(n)]
    live = list(range(n))
    for i in range(40):
        new = [f16(rng, n, h, d) for h in (h_q, h_kv, h_kv)]
        for x, y in zip((q, k, v), new):
            x.copy_(torch.from_numpy(y))
        for b in live:
            ks[b].append(new[1][b:b + 1])
            vs[b].append(new[2][b:b + 1])
        graph.replay()
        missing, whole, pages, sparse = (x.cpu().numpy() for x in results)
        assert missing[0] == 0
        tab, bn, sc = table.cpu().numpy(), bounds[0].cpu().numpy(), bounds[1].cpu().numpy()
        for b in live if i % 5 == 0 or i > 35 else ():
            kk, vv = held(np.concatenate(ks[b])), held(np.concatenate(vs[b]))
            pos = prompt + i
            assert (pages[b] == chosen64(new[0][b], h_kv, bn, sc, tab[b], pos, page, n_pages, 5, 1, 2)).all()
            for h in range(h_kv):
                rows = slice(4 * h, 4 * h + 4)
                y, tol = attended64(new[0][b, rows], kk[:, h], vv[:, h], d ** -0.5)
                assert (np.abs(whole[b, rows] - y) <= tol).all()
                tokens = [j for c in pages[b, h] if c >= 0 for j in range(c * page, min((c + 1) * page, pos + 1))]
                y, tol = attended64(new[0][b, rows], kk[tokens, h], vv[tokens, h], d ** -0.5)
                assert (np.abs(sparse[b, rows] - y) <= tol).all()
        if i == 20:                                                      # the second request is done; its row goes on as an empty one
            live.remove(1)
            cache.release(refs, table, dev(torch, [1]))
            kv_len[1] = -100
            moved = cache.compact(refs, table, bounds)
            alive = int((refs > 0).sum())
            assert (refs[:alive] > 0).all() and sorted(moved[moved >= 0].tolist()) == list(range(alive))
    assert cache.device_status() == (0, 0)


def test_other_streams_and_two_at_once(P, torch):
    """Calls on two streams with workspaces of their own, and through the Python half: the same bits."""
    rng = np.random.default_rng(12)
    cache, batch, kv, start, prefix = sharing(P, torch, [(900, [40, 300, 70, 9])], 16, 8, 128, 1, seed=6)
    b = cache.key_bounds()
    cache.summarise(b, *batch.whole, sum(batch.lens))
    q = torch.from_numpy(f16(rng, batch.T, 32, 128)).cuda()
    pages = cache.select(q, b, *batch.args, 20)
    want = cache.attention_shared(q, *batch.args, 1, start, prefix), cache.attention_selected(q, pages, *batch.args)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(10):
        for s in streams:
            got.append((cache.attention_shared(q, *batch.args, 1, start, prefix, stream=s), cache.attention_selected(q, cache.select(q, b, *batch.args, 20, stream=s), *batch.args, stream=s)))
    torch.cuda.synchronize()
    for a in got:
        assert torch.equal(a[0], want[0]) and torch.equal(a[1], want[1])


def test_workspaces_by_what_a_call_needs(P, torch):
    """Prompts, which do not share, take what attention takes; a batch over a long table more."""
    lib = P.lib
    cache = P.PagedKV(8, 16, 8, 128)
    plain = lib.qlinear_paged_attention_workspace(cache._h, 32, 4, 4000)
    assert lib.qlinear_paged_attention_shared_workspace(cache._h, 32, 300, 4, 16000, 4000, 0) == plain > 0
    assert lib.qlinear_paged_attention_shared_workspace(cache._h, 32, 4096, 64, 64, 1, 1) > 2 * 64 * 32 * 130 * 4
    assert lib.qlinear_paged_attention_shared_workspace(cache._h, 31, 300, 4, 4, 1, 1) == 0


# ---------------------------------------------------------------------------- read back by blocks
@pytest.mark.parametrize("h_kv,d,page", [(3, 128, 16), (2, 64, 64), (1, 256, 32)])
def test_read_of_many_rows(P, torch, h_kv, d, page):
    """Rows at every place of a block, before the first token, without a page, of no sequence; equal to the rows read a few at a time, bit for bit."""
    rng = np.random.default_rng(page)
    lens, new = [700, 33, 5, 901, 16], [695, 33, 40, 300, 16]
    batch = Batch(torch, lens, lens, page, seed=page)
    cache, kv = filled(P, torch, batch, h_kv, d)
    table = batch.table.copy()
    table[3, 700 // page], table[0, 1] = -1, batch.n_pages + 7
    starts = [4]
    for n in new:
        starts.append(starts[-1] + n)
    T = starts[-1] + 9
    args = dev(torch, table), dev(torch, lens), dev(torch, starts)
    got = [x.cpu().numpy() for x in cache.read(*args, T)]
    for b, (n, m) in enumerate(zip(lens, new)):
        for c in range(m):
            pos, t = n - m + c, starts[b] + c
            x = table[b, pos // page] if pos >= 0 else -1
            for y, whole in zip(got, kv[b]):
                want = whole[pos].astype(np.float16) if 0 <= x < batch.n_pages else np.zeros((h_kv, d), np.float16)
                assert (y[t] == want).all(), (b, pos)
        few = min(m, 20)
        for a, y in zip(cache.read(args[0][b:b + 1], args[1][b:b + 1], dev(torch, [0, few]), few), got):
            assert (a.cpu().numpy() == y[starts[b] + m - few:starts[b] + m]).all()


# ---------------------------------------------------------------------------- large numbers
def test_two_thousand_sequences_that_share(P, torch):
    """As many sequences as a call takes (with its groups), all of the calls on them; a sample of the rows against 64 bits."""
    rng = np.random.default_rng(21)
    h_q, h_kv, d, page = 4, 2, 64, 16
    groups = [(96, [int(n) for n in rng.integers(1, 40, 20)]) for _ in range(96)]
    cache, batch, kv, start, prefix = sharing(P, torch, groups, page, h_kv, d, [1 + b % 2 for b in range(1952)], seed=22, alone=[int(n) for n in rng.integers(1, 90, 32)])
    assert len(batch.lens) + len(groups) == 2048
    q = f16(rng, batch.T, h_q, d)
    dq = torch.from_numpy(q).cuda()
    rows = [r for r in batch.rows() if r[1] % 37 == 0 or r[1] > 1940]
    want, tol = attention64(q, kv, batch, d ** -0.5, rows=rows, max_q=10 ** 6)
    check(cache.attention_shared(dq, *batch.args, batch.max_q, start, prefix).cpu().numpy(), want, tol, rows)
    b = cache.key_bounds()
    cache.summarise(b, *batch.whole, sum(batch.lens))
    W = batch.table.shape[1]
    pages = cache.select(dq, b, *batch.args, W)                          # (every page)
    check(cache.attention_selected(dq, pages, *batch.args).cpu().numpy(), want, tol, rows)
    few = cache.select(dq, b, *batch.args, 3).cpu().numpy()
    bounds, scales = (x.cpu().numpy() for x in b)
    for t, s, pos in rows:
        assert (few[t] == chosen64(q[t], h_kv, bounds, scales, batch.table[s], pos, page, batch.n_pages, 3, 1, 1)).all()


@pytest.mark.parametrize("h_q,h_kv,d,page", [(64, 1, 128, 1024), (40, 40, 64, 16), (96, 2, 256, 64)])
def test_many_heads_that_share(P, torch, h_q, h_kv, d, page):
    """Many query heads a KV head, many KV heads, large pages: shared beginnings, lists, choices."""
    rng = np.random.default_rng(h_q)
    cache, batch, kv, start, prefix = sharing(P, torch, [(1100, [5, 90, 700]), (70, [3, 4])], page, h_kv, d, 1, seed=h_q, before=1, behind=1)
    q = f16(rng, batch.T, h_q, d)
    dq = torch.from_numpy(q).cuda()
    want, tol = attention64(q, kv, batch, d ** -0.5, max_q=10 ** 6)
    check(cache.attention_shared(dq, *batch.args, 1, start, prefix).cpu().numpy(), want, tol, batch.rows())
    b = cache.key_bounds()
    cache.summarise(b, *batch.whole, sum(batch.lens))
    bounds, scales = (x.cpu().numpy() for x in b)
    pages = cache.select(dq, b, *batch.args, 2, 1, 0)
    got, g = cache.attention_selected(dq, pages, *batch.args).cpu().numpy().astype(np.float64), h_q // h_kv
    pages = pages.cpu().numpy()
    for t, s, pos in batch.rows():
        assert (pages[t] == chosen64(q[t], h_kv, bounds, scales, batch.table[s], pos, page, batch.n_pages, 2, 1, 0)).all()
        for h in range(h_kv):
            tokens = [j for c in pages[t, h] if c >= 0 for j in range(c * page, min((c + 1) * page, pos + 1))]
            y, e = attended64(q[t, g * h:g * h + g], kv[s][0][tokens, h], kv[s][1][tokens, h], d ** -0.5)
            assert (np.abs(got[t, g * h:g * h + g] - y) <= e).all()


def test_a_prompt_over_listed_pages(P, torch):
    """Every row of a prompt with a list of its own: more segments than CTAs by far."""
    rng = np.random.default_rng(31)
    h_q, h_kv, d, page, n = 4, 2, 128, 32, 2500
    batch = Batch(torch, [n, 300], [n, 300], page)
    cache, kv = filled(P, torch, batch, h_kv, d)
    b = cache.key_bounds()
    cache.summarise(b, *batch.args, batch.T)
    q = f16(rng, batch.T, h_q, d)
    dq = torch.from_numpy(q).cuda()
    pages = cache.select(dq, b, *batch.args, 5, 1, 2)
    got, listed = cache.attention_selected(dq, pages, *batch.args).cpu().numpy().astype(np.float64), pages.cpu().numpy()
    for t, s, pos in batch.rows()[::29]:
        for h in range(h_kv):
            tokens = [j for c in listed[t, h] if c >= 0 for j in range(c * page, min((c + 1) * page, pos + 1))]
            y, e = attended64(q[t, 2 * h:2 * h + 2], kv[s][0][tokens, h], kv[s][1][tokens, h], d ** -0.5)
            assert (np.abs(got[t, 2 * h:2 * h + 2] - y) <= e).all()


def test_scores_of_millions(P, torch):
    """Large queries and scales: differences of scores are taken before they are scaled, in the join as well (weights of one token, the others vanish)."""
    rng = np.random.default_rng(32)
    cache, batch, kv, start, prefix = sharing(P, torch, [(900, [100, 40, 300])], 16, 2, 128, 1, seed=7)
    q = (f16(rng, batch.T, 8, 128).astype(np.float32) * 100).astype(np.float16)
    W = batch.table.shape[1]
    pages = dev(torch, np.broadcast_to(np.arange(W), (batch.T, 2, W)))
    apart = np.zeros((batch.T, 8), bool)                                 # heads whose largest score stays the largest whatever the keys' rounding (2^-11 of each product) does to two of them
    best = np.zeros((batch.T, 8, 128))
    for r, s, pos in batch.rows():
        for h in range(8):
            k = kv[s][0][:pos + 1, h // 4]
            x = k @ q[r, h].astype(np.float64)
            top = np.sort(x)[-2:]
            apart[r, h] = top[1] - top[0] > 2 * 2.0 ** -11 * (np.abs(k) @ np.abs(q[r, h]).astype(np.float64)).max() + 1
            best[r, h] = kv[s][1][x.argmax(), h // 4]
    assert apart.mean() > 0.5
    calls = lambda scale: (cache.attention_selected(torch.from_numpy(q).cuda(), pages, *batch.args, scale=scale), cache.attention_shared(torch.from_numpy(q).cuda(), *batch.args, 1, start, prefix, scale=scale))
    for scale in (1e3, 1e15):                                            # one token's weight is left: its value, rounded to fp16 with the weight's own rounding on the way
        for y in calls(scale):
            y = y.cpu().numpy().astype(np.float64)
            assert (np.abs(y - best) <= 4 * 2.0 ** -11 * np.abs(best))[apart].all() and np.isfinite(y).all()
    want, tol = attention64(q, kv, batch, 0.0, max_q=10 ** 6)
    for y in calls(0.0):
        check(y.cpu().numpy(), want, tol, batch.rows())


def test_rows_named_a_thousand_times_in_lists(P, torch):
    """q_start against the rules, so that the segments pass 32 bits: the kernel sees it and does nothing but zeros."""
    cache = P.PagedKV(8, 16, 1, 64)
    T, B = 70000, 2047
    q = torch.randn(T, 64, device="cuda").half()
    out = torch.full((T, 1, 64), 7.5, dtype=torch.float16, device="cuda")
    start = dev(torch, [0, T] * (B // 2) + [0, T])
    assert start.shape == (B + 1,)
    cache.attention_selected(q, torch.zeros((T, 1, 1), dtype=torch.int32, device="cuda"), torch.zeros((B, 1), dtype=torch.int32, device="cuda"), dev(torch, [16] * B), start, out=out)
    assert (out == 0).all() and cache.device_status() == (0, 0)


def test_sequences_named_a_thousand_times_that_share(P, torch):
    """group_start against the rules: a call that ends."""
    cache = P.PagedKV(8, 16, 1, 64)
    T, G = 1000000, 1023
    q = torch.randn(T, 64, device="cuda").half()
    out = cache.attention_shared(q, dev(torch, [list(range(8))] * 2), dev(torch, [600000] * 2), dev(torch, [0, T // 2, T]), 1, dev(torch, [0, 2] * (G // 2) + [0, 2]), dev(torch, [64] * G))
    assert out.shape == (T, 1, 64) and cache.device_status() == (0, 0)


# ---------------------------------------------------------------------------- refusals
def test_refused(P, torch):
    cache = P.PagedKV(8, 16, 2, 64)
    q, table, kv, start = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda"), dev(torch, [[0, 1], [2, 3]]), dev(torch, [3, 4]), dev(torch, [0, 1, 2])
    b, batch, pages = cache.key_bounds(), (table, kv, start), dev(torch, np.zeros((2, 2, 2)))
    group, prefix = dev(torch, [0, 2]), dev(torch, [16])
    shared = lambda q=q, batch=batch, max_q=1, group=group, prefix=prefix, **kw: cache.attention_shared(q, *batch, max_q, group, prefix, **kw)
    bad = [lambda: cache.summarise(b, table, kv[:1], start, 2), lambda: cache.summarise((b[0][:4], b[1]), *batch, 2), lambda: cache.summarise((b[0].short(), b[1]), *batch, 2), lambda: cache.summarise((b[0], b[1].cpu()), *batch, 2),
           lambda: cache.summarise(b, *batch, -1),
           lambda: cache.select(q[:, :3], b, *batch, 2), lambda: cache.select(q.float(), b, *batch, 2), lambda: cache.select(q, b, *batch, 0), lambda: cache.select(q, b, *batch, 2, 2, 1), lambda: cache.select(q, b, *batch, 2, -1, 1),
           lambda: cache.select(q, b, *batch, 2 ** 32 + 2), lambda: cache.select(q, b, *batch, 2, out=pages.long()), lambda: cache.select(q, b, *batch, 2, out=pages[:1]),
           lambda: cache.select(q, b, torch.zeros((2, 262145), dtype=torch.int32, device="cuda"), kv, start, 2),
           lambda: cache.attention_selected(q, pages[:, :1], *batch), lambda: cache.attention_selected(q, pages.long(), *batch), lambda: cache.attention_selected(q, pages.transpose(0, 1), table, kv, start[:2]),
           lambda: cache.attention_selected(q, pages, *batch, softcap=-1.0), lambda: cache.attention_selected(q, pages, *batch, scale=1e16), lambda: cache.attention_selected(q, pages, *batch, scale=float("nan")),
           lambda: cache.attention_selected(q, pages, *batch, out=q), lambda: cache.attention_selected(q[:, :3], pages, *batch),
           lambda: shared(max_q=-1), lambda: shared(group=group[:1]), lambda: shared(prefix=prefix.float()), lambda: shared(prefix=prefix.cpu()), lambda: shared(softcap=float("inf")), lambda: shared(scale=float("inf")),
           lambda: shared(out=q), lambda: shared(q=q[:, :3]), lambda: shared(group=dev(torch, [0] * 2049), prefix=dev(torch, [0] * 2048)), lambda: shared(max_q=2 ** 32 + 1)]
    for i, call in enumerate(bad):
        with pytest.raises(P.QLinearError) as e:
            call()
        assert e.value.status == P.QL_ERR_INVALID_ARG, i


def test_after_an_expired_wait(P, torch):
    """A wait of this unit's kernels reports through the device's word: the calls refuse until it has been read."""
    rng = np.random.default_rng(0)
    lin = P.QLinear.from_weights(rng.integers(-8, 8, (128, 64)).astype(np.int8), np.full((128, 2), 0.01, np.float16), 4, 32, device="cuda:0")
    cache = P.PagedKV(4, 16, 1, 64)
    refs, table, kv, start = dev(torch, [0] * 4), dev(torch, [[0, 1]]), dev(torch, [3]), dev(torch, [0, 1])
    q = torch.zeros((1, 1, 64), dtype=torch.float16, device="cuda")
    b = cache.key_bounds()
    lin.debug_expire_wait()
    torch.cuda.synchronize()
    calls = [lambda: cache.fork(refs, table, dev(torch, [0]), dev(torch, [3])), lambda: cache.release(refs, table, dev(torch, [0])), lambda: cache.reserve(refs, table, kv, start, 1), lambda: cache.compact(refs, table),
             lambda: cache.summarise(b, table, kv, start, 1), lambda: cache.select(q, b, table, kv, start, 1, 0), lambda: cache.attention_selected(q, dev(torch, [[[0]]]), table, kv, start),
             lambda: cache.attention_shared(q, table, kv, start, 1, dev(torch, [0, 1]), dev(torch, [0]))]
    for call in calls:
        with pytest.raises(P.QLinearError) as e:
            call()
        assert e.value.status == P.QL_ERR_DEVICE_TIMEOUT
    assert cache.device_status()[0] == P.QL_ERR_DEVICE_TIMEOUT and cache.device_status() == (0, 0)
    for call in calls:
        call()
    torch.cuda.synchronize()
