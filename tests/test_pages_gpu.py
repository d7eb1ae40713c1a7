"""Pages that requests share: page tables forked and released, pages reserved (a shared one copied before it is written), live pages moved together.  Whole numbers against
plain programs over lists, contents bit for bit."""
import numpy as np
import pytest

from test_paged_gpu import f16

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
    return torch.tensor(np.asarray(a, dtype=np.int32), dtype=torch.int32, device="cuda")


def forked(refs, table, parents, lengths, page):
    refs, W = list(refs), len(table[0])
    out = []
    for p, n in zip(parents, lengths):
        row = [int(table[p][j]) if 0 <= p < len(table) and j < -(-n // page) else -1 for j in range(W)]
        row = [x if 0 <= x < len(refs) else -1 for x in row]
        for x in row:
            if x >= 0:
                refs[x] += 1
        out.append(row)
    return out, refs


def reserved(refs, table, kv_len, starts, T, page):
    """(table, refs, missing, [(from, to, tokens)]) by a program on the host."""
    refs, table = list(refs), [list(r) for r in table]
    need = []
    for b, n in enumerate(kv_len):
        s, e = starts[b], starts[b + 1]
        rows = 0 if s < 0 or e > T or e < s else e - s
        if rows and n > 0:
            for j in range(max(n - rows, 0) // page, min((n - 1) // page + 1, len(table[b]))):
                x = table[b][j] if 0 <= table[b][j] < len(refs) else -1
                if x < 0 or refs[x] > 1:
                    need.append((b, j, x, max(max(n - rows, 0) - j * page, 0)))
    free = [x for x, c in enumerate(refs) if c == 0]
    if len(need) > len(free):
        return table, refs, len(need) - len(free), []
    copies = []
    for (b, j, x, older), to in zip(need, free):
        table[b][j] = to
        refs[to] = 1
        if x >= 0:
            refs[x] -= 1
            if older:
                copies.append((x, to, older))
    return table, refs, 0, copies


def compacted(refs, table):
    n = sum(c > 0 for c in refs)
    moved = [x if c > 0 else -1 for x, c in enumerate(refs)]
    for x, to in zip((x for x in range(n, len(refs)) if refs[x] > 0), (x for x in range(n) if refs[x] <= 0)):
        moved[x] = to
    new = [c if c <= 0 and x >= n else 0 for x, c in enumerate(refs)]
    for x, to in enumerate(moved):
        if to >= 0:
            new[to] = refs[x]
    return moved, new, [[moved[x] if 0 <= x < len(refs) else x for x in r] for r in table]


def full(P, torch, n_pages, page, h_kv, d, seed=0):
    """A cache whose every place holds a token, and its pages' bytes."""
    cache = P.PagedKV(n_pages, page, h_kv, d)
    cache.pool.copy_(torch.randint(0, 256, cache.pool.shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(seed)))
    return cache, cache.pool.clone()


def tokens_of(torch, cache, page, tokens):
    """(k, v) of the first tokens of a page."""
    one = lambda *a: dev(torch, a)
    return cache.read(one([page]), one(tokens), one(0, tokens), tokens)


def random_tables(rng, n_pages, B, W, share=0.3):
    """Page tables whose entries refs count: some pages in two rows, some entries without a page."""
    refs = np.zeros(n_pages, np.int32)
    table = np.full((B, W), -1, np.int32)
    order = list(rng.permutation(n_pages)[: n_pages * 2 // 3])
    for b in range(B):
        for j in range(W):
            if rng.random() < 0.15:
                table[b, j] = rng.choice([-1, n_pages, n_pages + 5, -7])
                continue
            used = np.flatnonzero(refs)
            x = rng.choice(used) if len(used) and rng.random() < share else order.pop() if order else -1
            table[b, j] = x
            if x >= 0:
                refs[x] += 1
    return refs, table


# ---------------------------------------------------------------------------- fork and release
@pytest.mark.parametrize("page,W", [(16, 1), (16, 7), (64, 300), (1024, 3)])
def test_fork(P, torch, page, W):
    rng = np.random.default_rng(W)
    refs, table = random_tables(rng, 500, 6, W)
    cache = P.PagedKV(500, page, 1, 64)
    parents = [0, 3, 3, -1, 6, 5, 2, 0, 2 ** 31 - 1]
    lengths = [page * W, 1, page + 1, 40, 40, 0, page * W * 3, -5, 9]
    want, want_refs = forked(refs, table, parents, lengths, page)
    r = dev(torch, refs)
    base = dev(torch, np.concatenate([table, np.full((len(parents), W), 77)]))   # children in other rows of the same array
    out = cache.fork(r, base[:6], dev(torch, parents), dev(torch, lengths), out=base[6:])
    assert out.data_ptr() == base[6:].data_ptr() and (out.cpu().numpy() == want).all() and (r.cpu().numpy() == want_refs).all()
    assert (base[:6].cpu().numpy() == table).all()
    r = dev(torch, refs)
    wide = dev(torch, np.pad(table, ((0, 0), (0, 3))))[:, :W]             # (a stride)
    assert (cache.fork(r, wide, dev(torch, parents), dev(torch, lengths)).cpu().numpy() == want).all() and (r.cpu().numpy() == want_refs).all()


def test_fork_and_release_of_nothing(P, torch):
    cache = P.PagedKV(4, 16, 1, 64)
    refs, none = dev(torch, [1, 0, 0, 0]), dev(torch, [])
    table = dev(torch, [[0, -1]])
    assert cache.fork(refs, table, none, none).shape == (0, 2)
    cache.release(refs, table, none)
    assert cache.fork(refs, table[:, :0], dev(torch, [0]), dev(torch, [5])).shape == (1, 0)
    assert refs.tolist() == [1, 0, 0, 0] and table.tolist() == [[0, -1]]


@pytest.mark.parametrize("W", [1, 7, 700])
def test_release(P, torch, W):
    rng = np.random.default_rng(W)
    page = 32
    refs, table = random_tables(rng, 900, 8, W)
    cache = P.PagedKV(900, page, 1, 64)
    rows, keep = [5, 1, 5, -1, 8, 0, 7], [page * 2, 0, page + 1, 0, 0, page * W, -3]
    want, want_refs = table.copy(), refs.copy()
    for b in range(8):
        kept = min([-(-max(k, 0) // page) for r, k in zip(rows, keep) if r == b] + [W])
        for x in want[b, kept:]:
            if 0 <= x < 900:
                want_refs[x] -= 1
        want[b, kept:] = -1
    r, t = dev(torch, refs), dev(torch, table)
    cache.release(r, t, dev(torch, rows), dev(torch, keep))
    assert (t.cpu().numpy() == want).all() and (r.cpu().numpy() == want_refs).all()
    cache.release(r, t, dev(torch, list(range(8))))
    assert (t.cpu().numpy() == -1).all() and (r.cpu().numpy() == 0).all()


# ---------------------------------------------------------------------------- reserve
CASES = [  # heads, d, page, sequences, pages, new tokens
    (2, 128, 16, 5, 60, 1), (1, 64, 64, 40, 300, 1), (4, 256, 32, 3, 40, 70), (3, 64, 128, 7, 60, 129), (1, 64, 16, 200, 9000, 40), (1, 64, 16, 2, 40000, 9000), (8, 128, 64, 60, 600, 30)]


@pytest.mark.parametrize("h_kv,d,page,B,n_pages,new", CASES)
@pytest.mark.parametrize("spare", [0, 3, -2])
def test_reserve(P, torch, h_kv, d, page, B, n_pages, new, spare):
    """Free pages in order, copies of what is shared, nothing at all when the pool is short."""
    rng = np.random.default_rng(B * new + spare + 2)
    held = [int(rng.integers(0, 5 * page)) for _ in range(B)]
    held[0] = 2 * page                                                   # (new tokens begin a page)
    W = (max(held) + new) // page + 2
    starts = [2]
    for b in range(B):
        starts.append(starts[-1] + (0 if b % 5 == 3 else int(rng.integers(1, new + 1))))
    kv_len = [held[b] + starts[b + 1] - starts[b] for b in range(B)]
    T = starts[-1] + 3
    refs, table = np.zeros(n_pages, np.int64), np.full((B, W), -1, np.int64)
    order = list(rng.permutation(n_pages))
    for b in range(B):
        for j in range(-(-held[b] // page)):
            table[b, j] = table[b - 1, j] if b % 3 == 1 and table[b - 1, j] >= 0 else order.pop()
            refs[table[b, j]] += 1
    _, _, short, _ = reserved(np.maximum(refs, 1), table, kv_len, starts, T, page)
    free = np.flatnonzero(refs == 0)
    refs[rng.permutation(free)[: len(free) - short - spare]] = 1          # (held by other tables: the pool has what is needed, three more, two too few)
    want, want_refs, missing, copies = reserved(refs, table, kv_len, starts, T, page)
    assert missing == max(0, -spare) and (len(copies) > 0 or spare < 0 or B < 40)
    cache, before = full(P, torch, n_pages, page, h_kv, d)
    r, t = dev(torch, refs), dev(torch, table)
    got = cache.reserve(r, t, dev(torch, kv_len), dev(torch, starts), T)
    assert got.tolist() == [missing] and (t.cpu().numpy() == want).all() and (r.cpu().numpy() == want_refs).all()
    written = [to for _, to, _ in copies]
    same = np.setdiff1d(np.arange(n_pages), written)
    assert torch.equal(cache.pool[same.tolist()], before[same.tolist()])
    for x, to, older in copies[:20]:
        for a, b in zip(tokens_of(torch, cache, x, older), tokens_of(torch, cache, to, older)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_reserve_lengths_at_the_edge(P, torch):
    """Empty sequences, lengths below zero and beyond the table, rows that are none of the call's, rows before the first token."""
    cache = P.PagedKV(50, 16, 1, 64)
    kv_len = [0, -5, -2 ** 31, 100, 2 ** 31 - 1, 3, 20, 16, 1]
    starts = [0, 2, 4, 6, 9, 10, 18, 19, 20, 40]                          # (the last one's rows are not in the call; sequence 5 has 8 rows and 3 tokens)
    table = np.full((9, 4), -1)
    want, want_refs, missing, _ = reserved([0] * 50, table, kv_len, starts, 30, 16)
    assert missing == 0
    r, t = dev(torch, [0] * 50), dev(torch, table)
    assert cache.reserve(r, t, dev(torch, kv_len), dev(torch, starts), 30).tolist() == [0]
    assert t.cpu().tolist() == want and r.cpu().tolist() == want_refs
    none = dev(torch, [])
    assert cache.reserve(r, t[:0], none, dev(torch, [0]), 0).tolist() == [0]
    assert cache.reserve(r, t[:, :0], dev(torch, kv_len), dev(torch, starts), 30).tolist() == [0]
    assert r.cpu().tolist() == want_refs


# ---------------------------------------------------------------------------- compact
@pytest.mark.parametrize("h_kv,d,page,n_pages", [(2, 128, 16, 1), (1, 64, 16, 127), (3, 64, 64, 128), (2, 256, 32, 129), (1, 64, 16, 5000), (8, 128, 64, 700), (1, 64, 16, 33001)])
@pytest.mark.parametrize("live", [0.0, 0.5, 0.97, 1.0])
def test_compact(P, torch, h_kv, d, page, n_pages, live):
    rng = np.random.default_rng(n_pages)
    B, W = 5, 40
    refs = np.where(rng.random(n_pages) < live, rng.integers(1, 4, n_pages), 0)
    table = rng.integers(-3, n_pages + 3, (B, W))                         # (entries of free pages among them)
    moved, new_refs, new_table = compacted(refs.tolist(), table.tolist())
    cache, before = full(P, torch, n_pages, page, h_kv, d)
    bounds = cache.key_bounds()
    bounds[0].copy_(torch.randint(-127, 128, bounds[0].shape, dtype=torch.int8))
    bounds[1].copy_(torch.rand(bounds[1].shape))
    kept = [b.clone() for b in bounds]
    r, t = dev(torch, refs), dev(torch, table)
    got = cache.compact(r, t, bounds)
    assert got.tolist() == moved and r.tolist() == new_refs and t.tolist() == new_table
    old = [x for x in range(n_pages) if moved[x] >= 0]
    new = [moved[x] for x in old]
    for a, b in ((cache.pool, before), (bounds[0], kept[0]), (bounds[1], kept[1])):
        assert torch.equal(a[new], b[old])
    again = cache.compact(r, t)                                          # nothing is left to move
    assert again.tolist() == [x if c > 0 else -1 for x, c in enumerate(new_refs)] and t.tolist() == new_table and torch.equal(cache.pool[new], before[old])


def test_two_thousand_sequences(P, torch):
    """As many sequences as the calls take: forked from 7, written apart, given back."""
    rng = np.random.default_rng(8)
    n_pages, page, W = 9000, 16, 6
    refs, table = np.zeros(n_pages, np.int64), np.full((7, W), -1, np.int64)
    lens = [1, 16, 40, 17, 64, 33, 80]
    order = rng.permutation(n_pages)
    for b, n in enumerate(lens):
        k = -(-n // page)
        table[b, :k] = order[10 * b:10 * b + k]
        refs[table[b, :k]] = 1
    parents = rng.integers(0, 7, 2048)
    held = [lens[p] for p in parents]
    want, want_refs = forked(refs, table, parents, held, page)
    cache, before = full(P, torch, n_pages, page, 1, 64)
    r = dev(torch, refs)
    t = cache.fork(r, dev(torch, table), dev(torch, parents), dev(torch, held))
    assert t.tolist() == want and r.tolist() == want_refs
    kv_len = [n + 1 + i % 3 for i, n in enumerate(held)]
    starts = np.concatenate([[0], np.cumsum([1 + i % 3 for i in range(2048)])]).tolist()
    want, want_refs, missing, copies = reserved(want_refs, want, kv_len, starts, starts[-1], page)
    assert missing == 0 and len(copies) > 1000
    assert cache.reserve(r, t, dev(torch, kv_len), dev(torch, starts), starts[-1]).tolist() == [0]
    assert t.tolist() == want and r.tolist() == want_refs
    assert all(torch.equal(cache.pool[to], before[x]) for x, to, _ in copies[::41])
    rows = rng.permutation(2048)[:2000]
    cache.release(r, t, dev(torch, rows))
    for b in rows:
        for x in want[b]:
            if x >= 0:
                want_refs[x] -= 1
    assert r.tolist() == want_refs


# ---------------------------------------------------------------------------- refusals
def test_refused(P, torch):
    cache = P.PagedKV(8, 16, 2, 64)
    refs, table = dev(torch, [1] * 8), dev(torch, [[0, 1], [2, 3]])
    kv, start, rows = dev(torch, [3, 4]), dev(torch, [0, 1, 2]), dev(torch, [0])
    cpu = lambda t: t.cpu()
    bad = [lambda: cache.fork(refs[:7], table, rows, rows), lambda: cache.fork(refs, table, rows, kv), lambda: cache.fork(refs, table.long(), rows, rows), lambda: cache.fork(refs, cpu(table), rows, rows),
           lambda: cache.fork(refs, table, rows, rows, out=table[:1]), lambda: cache.fork(refs, table, rows, rows, out=table[:, :1]), lambda: cache.fork(refs, table.t(), rows, rows),
           lambda: cache.fork(refs, table, dev(torch, [0] * 2049), dev(torch, [0] * 2049)),
           lambda: cache.release(refs.float(), table, rows), lambda: cache.release(refs, table, rows, kv), lambda: cache.release(refs, table[0], rows), lambda: cache.release(refs, table, rows.long()),
           lambda: cache.reserve(refs, table, kv[:1], start, 2), lambda: cache.reserve(refs, table, kv, start, -1), lambda: cache.reserve(refs[::2], table, kv, start, 2), lambda: cache.reserve(refs, table, kv, start, 2 ** 32 + 2),
           lambda: cache.compact(cpu(refs), table), lambda: cache.compact(refs, table, (cache.key_bounds()[0][:4], cache.key_bounds()[1])), lambda: cache.compact(refs, table, (cache.key_bounds()[0].float(), cache.key_bounds()[1]))]
    for i, call in enumerate(bad):
        with pytest.raises(P.QLinearError) as e:
            call()
        assert e.value.status == P.QL_ERR_INVALID_ARG, i
    assert refs.tolist() == [1] * 8 and table.tolist() == [[0, 1], [2, 3]]


def test_the_python_half_does_the_same(P, torch):
    """A call with a stream goes through ctypes: the same results, and another stream."""
    rng = np.random.default_rng(5)
    refs, table = random_tables(rng, 200, 4, 9)
    args = dev(torch, [0, 2, 3]), dev(torch, [40, 100, 70])
    kv, starts, rows = dev(torch, [43, 101, 75]), dev(torch, [0, 3, 4, 9]), dev(torch, [1])
    results = []
    for stream in (None, torch.cuda.Stream()):
        cache, _ = full(P, torch, 200, 16, 2, 128)
        r, t = dev(torch, refs), dev(torch, table)
        torch.cuda.synchronize()
        kw = {} if stream is None else {"stream": stream}
        child = cache.fork(r, t, *args, **kw)
        missing = cache.reserve(r, child, kv, starts, 9, **kw)
        cache.release(r, t, rows, **kw)
        bounds = cache.key_bounds()
        torch.cuda.synchronize()
        cache.summarise(bounds, child, kv, starts, 9, **kw)
        moved = cache.compact(r, child, bounds, **kw)
        torch.cuda.synchronize()
        results.append([r, t, child, missing, moved, *bounds, cache.pool[(moved[moved >= 0]).long().sort().values]])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_captured_calls_follow_the_arrays(P, torch):
    """A captured fork, reserve, release and compact act on what the arrays hold when it is replayed."""
    rng = np.random.default_rng(6)
    cache, before = full(P, torch, 300, 16, 1, 64)
    r, t = dev(torch, [0] * 300), dev(torch, np.full((4, 9), -1))
    parents, lengths, kv, starts, rows = dev(torch, [0, 0]), dev(torch, [0, 0]), dev(torch, [0, 0]), dev(torch, [0, 1, 2]), dev(torch, [3])
    child = torch.empty((2, 9), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(2):
            cache.fork(r, t, parents, lengths, out=child)
            cache.reserve(r, child, kv, starts, 2)
            cache.release(r, t, rows)
            cache.compact(r, child)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.fork(r, t, parents, lengths, out=child)
        missing = cache.reserve(r, child, kv, starts, 2)
        cache.release(r, t, rows)
        moved = cache.compact(r, child)
    for trial in range(3):
        refs, table = random_tables(rng, 300, 4, 9)
        n = [int(x) for x in rng.integers(1, 120, 2)]
        cache.pool.copy_(before)
        for a, b in ((r, refs), (t, table), (parents, [trial, 2]), (lengths, n), (kv, [x + 1 for x in n]), (rows, [trial + 1])):
            a.copy_(dev(torch, b))
        g.replay()
        want, want_refs = forked(refs, table, [trial, 2], n, 16)
        want, want_refs, short, _ = reserved(want_refs, want, [x + 1 for x in n], [0, 1, 2], 2, 16)
        for x in table[trial + 1]:
            if 0 <= x < 300:
                want_refs[x] -= 1
        want_moved, want_refs, want = compacted(want_refs, want)
        assert missing.tolist() == [short] and moved.tolist() == want_moved and r.tolist() == want_refs and child.tolist() == want
