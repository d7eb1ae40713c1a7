"""The paged 4-bit cache: append with the rotation, read back, attention, against plain implementations in 64 bits (numpy)."""
import numpy as np
import pytest

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


def quantised(x):
    """What the cache holds of x [..., d] (fp16): integers and fp16 scales, by the stated IEEE operations."""
    x = x.astype(np.float32).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    s = np.minimum((np.abs(x).max(-1) / np.float32(7)).astype(np.float16), np.float16(9352))
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.clip(np.rint(x / s.astype(np.float32)[..., None]), -7, 7)
    return np.where(s[..., None] == 0, 0, q), s


def held(x):
    q, s = quantised(x)
    return (q * s.astype(np.float64)[..., None]).reshape(x.shape)


def rotated(x, cos, sin, rot, interleaved):
    """x fp16 [T, heads, d]; cos, sin fp32 [T, rot / 2]: each product and sum rounded to fp32, the result to fp16."""
    x32, y, c, s = x.astype(np.float32), x.copy(), cos[:, None], sin[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a], y[..., b] = x32[..., a] * c - x32[..., b] * s, x32[..., b] * c + x32[..., a] * s
    return y


class Batch:
    """Sequences of the given lengths with their last rows new, pages in random order, rows of padding around them."""

    def __init__(self, torch, lens, new, page, seed=0, before=0, behind=0, spare=2):
        rng = np.random.default_rng(seed)
        self.lens, self.new, self.page = lens, [min(n, l) for n, l in zip(new, lens)], page
        pages = [-(-n // page) for n in lens]
        self.n_pages = sum(pages) + spare
        order = rng.permutation(self.n_pages)
        W = max(pages + [1])
        self.table = np.full((len(lens), W), -1, np.int32)
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.starts = before + np.concatenate([[0], np.cumsum(self.new)])
        self.T = int(self.starts[-1]) + behind
        dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
        self.args = dev(self.table), dev(lens), dev(self.starts)
        self.whole = dev(self.table), dev(lens), dev(np.concatenate([[0], np.cumsum(lens)]))
        self.max_q = max(self.new + [1])

    def rows(self):
        """(row, sequence, position) of every new token."""
        return [(int(self.starts[b]) + i, b, self.lens[b] - n + i) for b, n in enumerate(self.new) for i in range(n)]


def f16(rng, *shape):
    return rng.standard_normal(shape).astype(np.float16)


def filled(P, torch, batch, h_kv, d, seed=1, k_scale=1.0):
    """A cache that holds the batch's sequences, and what it stands for [sequence] -> (k, v) [len, h_kv, d] in 64 bits."""
    rng = np.random.default_rng(seed)
    n = sum(batch.lens)
    k, v = (f16(rng, n, h_kv, d) * np.float16(k_scale)).astype(np.float16), f16(rng, n, h_kv, d)
    cache = P.PagedKV(batch.n_pages, batch.page, h_kv, d)
    cache.append(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), *batch.whole)
    ends = np.cumsum(batch.lens)
    return cache, [(held(k[e - l:e]), held(v[e - l:e])) for e, l in zip(ends, batch.lens)]


def attention64(q, kv, batch, scale, softcap=0.0, window=0, rows=None, max_q=None):
    """(out, bound per element): the definition in 64 bits.  Beyond 48, 32, 24 rows per KV head (d 64, 128, 256) the keys are rounded to fp16(q s) as well: 2^-11 of each product.  The kernels round the unnormalised weights to fp16 (2^-11 relative, 2^-25 absolute below 2^-14,
    of weights whose largest is at least 1), the values q s to fp16 (2^-11) and the result (2^-11, 2^-25 absolute); scores are sums of d products in fp32 whose
    error moves a weight by exp(error) - 1."""
    T, h_q, d = q.shape
    out, tol = np.zeros((T, h_q, d)), np.zeros((T, h_q, d))
    g = h_q // kv[0][0].shape[1]
    key = 2.0 ** -11 if (max_q or batch.max_q) * g > {64: 48, 128: 32, 256: 24}[d] else 0.0
    for t, b, pos in rows or batch.rows():
        k, v = kv[b]
        lo, hi = (max(0, pos - window + 1) if window else 0), min(pos + 1, len(k))
        if hi <= lo:
            continue
        for hk in range(h_q // g):
            kk, vv = k[lo:hi, hk], v[lo:hi, hk]
            q64 = q[t, hk * g:(hk + 1) * g].astype(np.float64)
            x = q64 @ kk.T * scale
            dx = (key + (d + 40) * 2.0 ** -24) * (np.abs(q64) @ np.abs(kk).T) * abs(scale)         # sums in any order, scale, scores on a base-2 scale
            if softcap:
                x = softcap * np.tanh(x / softcap)
                dx = dx + 16 * 2.0 ** -24 * softcap                      # (quotient, exponential and reciprocal of a few ulp on numbers up to softcap)
            w = np.exp(x - x.max(-1, keepdims=True))
            p = w / w.sum(-1, keepdims=True)
            rel = np.expm1(dx + 2.0 ** -21 * (1 + np.abs(x - x.max(-1, keepdims=True)))).max(-1, keepdims=True)   # (the exponential's own ulps, its argument's rounding)
            y = p @ vv
            a = p @ np.abs(vv)
            e = (2 * rel + 2 * 2.0 ** -11 + (hi - lo) * 2.0 ** -24) * a + 2.0 ** -25 / w.sum(-1, keepdims=True) * np.abs(vv).sum(0)
            out[t, hk * g:(hk + 1) * g] = y
            tol[t, hk * g:(hk + 1) * g] = 1.01 * e + 2.0 ** -11 * np.abs(y) + 2.0 ** -25
    return out, tol


def check(out, want, tol, rows):
    for t, _, _ in rows:
        err = np.abs(out[t].astype(np.float64) - want[t])
        assert (err <= tol[t]).all(), (t, err.max(), tol[t].flat[err.argmax()])


HEADS = [(32, 8, 128), (8, 4, 256), (14, 2, 64), (4, 4, 64), (12, 1, 128)]


# ---------------------------------------------------------------------------- append and read
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_append_is_exact(P, torch, h_q, h_kv, d, page):
    """Turned queries and what the cache stands for, bit for bit: half and neighbouring pairs, all and part of the head, ragged new tokens."""
    rng = np.random.default_rng(d + page)
    batch = Batch(torch, [1, 37, 16, 200, 5], [1, 5, 16, 130, 0], page, seed=page, before=2, behind=3)
    n_pos = 150                                                          # (positions beyond the tables take the last row's angles)
    for rot in {d, d // 2, 32, 16}:
        ang = np.outer(np.arange(n_pos), 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot))
        cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
        for interleaved in (False, True):
            q, k, v = (f16(rng, batch.T, h, d) for h in (h_q, h_kv, h_kv))
            k[3, 0, :32] = 0                                             # a group of zeros
            cache = P.PagedKV(batch.n_pages, page, h_kv, d)
            dev = [torch.from_numpy(a).cuda() for a in (q, k, v, cos, sin)]
            mark = torch.full_like(dev[0], 7.5)
            got = cache.append(dev[1], dev[2], *batch.args, q=dev[0], cos=dev[3], sin=dev[4], interleaved=interleaved, q_out=mark)
            assert got is mark
            got_k, got_v = cache.read(*batch.args, batch.T)
            got, got_k, got_v = got.cpu().numpy(), got_k.cpu().numpy(), got_v.cpu().numpy()
            rows = batch.rows()
            t = [r[0] for r in rows]
            at = np.minimum([r[2] for r in rows], n_pos - 1)
            assert (got[t] == rotated(q[t], cos[at], sin[at], rot, interleaved)).all()
            assert (got_k[t] == held(rotated(k[t], cos[at], sin[at], rot, interleaved)).astype(np.float16)).all()
            assert (got_v[t] == held(v[t]).astype(np.float16)).all()
            rest = np.setdiff1d(np.arange(batch.T), t)
            assert (got[rest] == 7.5).all()


@pytest.mark.parametrize("n", [45, 700])
def test_append_token_by_token_equals_at_once(P, torch, n):
    """The bytes of the pool do not depend on how tokens came: one call, or one call per token; rows of a q/k/v projection, in place."""
    rng = np.random.default_rng(3)
    h_q, h_kv, d = 8, 2, 128
    batch = Batch(torch, [n], [n], 32)
    qkv = torch.from_numpy(f16(rng, n, (h_q + 2 * h_kv) * d)).cuda()
    cut = lambda x: (x[:, :h_q * d], x[:, h_q * d:(h_q + h_kv) * d], x[:, (h_q + h_kv) * d:])
    cos, sin = P.qlinear_rope_tables(n, d, device="cuda")
    a, b = (P.PagedKV(batch.n_pages, 32, h_kv, d) for _ in range(2))
    whole = qkv.clone()
    q, k, v = cut(whole)
    assert a.append(k, v, *batch.args, q=q, cos=cos, sin=sin, q_out=q) is q
    for i in range(n):
        q1, k1, v1 = cut(qkv[i:i + 1])
        y = b.append(k1, v1, batch.args[0], batch.args[1] * 0 + i + 1, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), q=q1, cos=cos, sin=sin)
        assert torch.equal(y, q[i:i + 1])
    assert torch.equal(a.pool, b.pool)


@pytest.mark.parametrize("T0", [0, 3, 13])
@pytest.mark.parametrize("h_kv,d", [(2, 128), (4, 256), (3, 64)])
def test_prompts_behind_what_is_there(P, torch, T0, h_kv, d):
    """Many rows behind tokens that the pages hold already: those stay, to the byte."""
    rng = np.random.default_rng(T0 + d)
    lens = [T0 + 600, T0 + 17, T0 + 1, T0 + 333]
    batch = Batch(torch, lens, [n - T0 for n in lens], 32, seed=T0)
    n = sum(lens)
    k, v = f16(rng, n, h_kv, d), f16(rng, n, h_kv, d)
    starts = np.concatenate([[0], np.cumsum(lens)])
    cache = P.PagedKV(batch.n_pages, 32, h_kv, d)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    old = np.concatenate([np.arange(s, s + T0) for s in starts[:-1]]).astype(int)
    new = np.concatenate([np.arange(s + T0, s + l) for s, l in zip(starts, lens)])
    if T0:
        cache.append(torch.from_numpy(k[old]).cuda(), torch.from_numpy(v[old]).cuda(), batch.args[0], i32([T0] * 4), i32(np.arange(5) * T0))
    cache.append(torch.from_numpy(k[new]).cuda(), torch.from_numpy(v[new]).cuda(), *batch.args)
    got_k, got_v = cache.read(*batch.whole, n)
    assert (got_k.cpu().numpy() == held(k).astype(np.float16)).all() and (got_v.cpu().numpy() == held(v).astype(np.float16)).all()


def test_append_equals_rotation_then_append_without(P, torch):
    rng = np.random.default_rng(4)
    batch = Batch(torch, [70, 9], [70, 9], 16)
    k, v = (torch.from_numpy(f16(rng, batch.T, 4, 64)).cuda() for _ in range(2))
    cos, sin = P.qlinear_rope_tables(128, 64, device="cuda")
    a, b = (P.PagedKV(batch.n_pages, 16, 4, 64) for _ in range(2))
    a.append(k, v, *batch.args, cos=cos, sin=sin)
    turned = b.append(torch.zeros_like(k), v, *batch.args, q=k, cos=cos, sin=sin)          # (k as queries, zeros as keys)
    b.append(turned, v, *batch.args)
    assert torch.equal(a.pool, b.pool)


@pytest.mark.parametrize("value", [65504.0, 6e-8, 1e-3, 0.0])
def test_extreme_groups(P, torch, value):
    """The largest fp16 number (the scale is held at 9352), the smallest (a scale that rounds to zero), and none but zeros."""
    x = np.zeros((1, 1, 64), np.float16)
    x[0, 0, 5] = value
    x[0, 0, 40:50] = -np.float16(value)
    batch = Batch(torch, [1], [1], 16)
    cache = P.PagedKV(batch.n_pages, 16, 1, 64)
    t = torch.from_numpy(x).cuda()
    cache.append(t, t, *batch.args)
    for got in cache.read(*batch.args, 1):
        got = got.cpu().numpy()
        assert (got == held(x).astype(np.float16)).all() and np.isfinite(got).all()
        if value == 65504:
            assert got[0, 0, 5] == 65464
        if value in (0, 6e-8):
            assert not got.any()


def test_places_outside_the_pool(P, torch):
    """Entries of the table outside the pool, and tokens behind the table's end: not stored, read as zeros, not attended to; nothing else changes."""
    rng = np.random.default_rng(6)
    batch = Batch(torch, [64, 64], [64, 64], 16, spare=0)
    k, v, q = (torch.from_numpy(f16(rng, 128, 2, 64)).cuda() for _ in range(3))
    cache = P.PagedKV(batch.n_pages, 16, 2, 64)
    table = batch.args[0].clone()
    kv = [(held(k.cpu().numpy()[s]), held(v.cpu().numpy()[s])) for s in (slice(0, 64), slice(64, 128))]
    for bad in (-1, batch.n_pages, 2 ** 31 - 1, -2 ** 31):
        table[0, 1] = bad
        cache.pool.zero_()
        cache.append(k, v, table, *batch.args[1:])
        assert not cache.pool[int(batch.table[0, 1])].any()
        got_k, got_v = cache.read(table, *batch.args[1:], 128)
        assert not got_k[16:32].any() and not got_v[16:32].any() and got_k[32:].any(-1).all()
        keep = np.r_[0:16, 32:64]
        for max_q, rows in ((64, (5, 20, 40, 63)), (1, (63,))):          # (every row at once; the last one alone)
            starts = batch.args[2] if max_q == 64 else torch.tensor([63, 64, 64], dtype=torch.int32, device="cuda")
            out = cache.attention(q, table, batch.args[1], starts, max_q).cpu().numpy()
            for t in rows:                                               # (the rows' own visible tokens without the lost ones)
                x = kv[0][0][:, 0] @ q[t, 0].cpu().numpy().astype(np.float64) / 8
                see = keep[keep <= t]
                w = np.exp(x[see] - x[see].max())
                want = w @ kv[0][1][see, 0] / w.sum()
                assert np.abs(out[t, 0] - want).max() < 2e-3 * np.abs(kv[0][1]).max()
    cache.pool.zero_()
    cache.append(k, v, batch.args[0][:, :2].contiguous(), *batch.args[1:])                  # a table that ends early
    got_k, _ = cache.read(*batch.args, 128)
    assert got_k[:32].any(-1).all() and not got_k[32:64].any() and got_k[64:96].any(-1).all() and not got_k[96:].any()


# ---------------------------------------------------------------------------- attention
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("page", [16, 128])
def test_decode(P, torch, h_q, h_kv, d, page):
    """One token of every sequence: lengths from one to long, ragged; the rows of padding stay."""
    lens = [1, 2, 15, 16, 17, 31, 129, 700, 2049, 0, 333]
    batch = Batch(torch, lens, [1] * len(lens), page, seed=d, before=1, behind=2)
    cache, kv = filled(P, torch, batch, h_kv, d)
    q = f16(np.random.default_rng(7), batch.T, h_q, d) * np.float16(2)
    out = torch.full((batch.T, h_q, d), 9.0, dtype=torch.float16, device="cuda")
    got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, 1, out=out).cpu().numpy()
    want, tol = attention64(q, kv, batch, d ** -0.5)
    check(got, want, tol, batch.rows())
    assert (got[0] == 9).all() and (got[-2:] == 9).all()


@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("new", [2, 5, 33, 150])
@pytest.mark.parametrize("softcap,window", [(0.0, 0), (30.0, 0), (0.0, 40), (50.0, 7)])
def test_rows_caps_and_windows(P, torch, h_q, h_kv, d, new, softcap, window):
    lens = [400, 150, 3, 77] if new == 150 else [new, 300, 64]
    batch = Batch(torch, lens, [new] * len(lens), 32, seed=new, behind=1)
    cache, kv = filled(P, torch, batch, h_kv, d)
    q = f16(np.random.default_rng(8), batch.T, h_q, d) * np.float16(2)
    out = torch.full((batch.T, h_q, d), 9.0, dtype=torch.float16, device="cuda")
    got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, batch.max_q, softcap=softcap, window=window, out=out).cpu().numpy()
    want, tol = attention64(q, kv, batch, d ** -0.5, softcap, window)
    check(got, want, tol, batch.rows())
    assert (got[-1] == 9).all()


@pytest.mark.parametrize("new", [1, 40])
def test_scale_strides_and_large_scores(P, torch, new):
    """A scale of the caller's, rows cut from wider ones, scores far apart (the maximum is raised many times), negative scale."""
    batch = Batch(torch, [777, 50], [new, new], 16)
    cache, kv = filled(P, torch, batch, 2, 128, k_scale=6)
    wide = torch.from_numpy(f16(np.random.default_rng(9), batch.T, 12 * 128) * np.float16(3)).cuda()
    q = wide[:, 128:9 * 128]
    for scale in (0.1, -0.05, 0.0):
        out = torch.zeros((batch.T, 10, 128), dtype=torch.float16, device="cuda")
        got = cache.attention(q, *batch.args, new, scale=scale, out=out[:, 1:9]).cpu().numpy()
        want, tol = attention64(q.cpu().numpy().reshape(batch.T, 8, 128), kv, batch, scale)
        check(got, want, tol, batch.rows())
        assert not out[:, 0].any() and not out[:, 9].any()


@pytest.mark.parametrize("more", [0, 100])
def test_more_rows_than_tokens(P, torch, more):
    """Rows whose positions lie before the sequence's first token, and sequences of no tokens: zeros."""
    lens, new = [2, 0, 5], [4, 2, 1 + more]
    starts = np.concatenate([[0], np.cumsum(new)])
    batch = Batch(torch, lens, [0, 0, 0], 16)
    cache, kv = filled(P, torch, batch, 2, 64)
    T = int(starts[-1])
    q = torch.from_numpy(f16(np.random.default_rng(2), T, 4, 64)).cuda()
    got = cache.attention(q, batch.args[0], batch.args[1], torch.tensor(starts, dtype=torch.int32, device="cuda"), max(new)).cpu().numpy()
    rows = [(int(starts[b]) + i, b, lens[b] - n + i) for b, n in enumerate(new) for i in range(n)]
    seen = [r for r in rows if r[2] >= 0]
    assert not got[[r[0] for r in rows if r[2] < 0]].any() and got[[r[0] for r in seen]].any(-1).all()
    want, tol = attention64(q.cpu().numpy(), kv, batch, 0.125, rows=seen, max_q=max(new))
    check(got, want, tol, seen)


@pytest.mark.parametrize("new,most", [(6, 4), (90, 70)])
def test_rows_behind_max_q_stay(P, torch, new, most):
    batch = Batch(torch, [140, 140], [new, new], 16)
    cache, kv = filled(P, torch, batch, 2, 64)
    q = f16(np.random.default_rng(2), 2 * new, 2, 64)
    out = torch.full((2 * new, 2, 64), 3.0, dtype=torch.float16, device="cuda")
    got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, most, out=out).cpu().numpy()
    want, tol = attention64(q, kv, batch, 0.125, max_q=most)
    check(got, want, tol, [r for r in batch.rows() if r[0] % new < most])
    assert (got[[t for t in range(2 * new) if t % new >= most]] == 3).all()


@pytest.mark.parametrize("max_q", [1, 64])
def test_rows_that_are_no_rows(P, torch, max_q):
    """q_start that runs backwards or leaves the call's rows: such a sequence has no rows; the others are served."""
    batch = Batch(torch, [20, 20, 20], [1, 1, 1], 16)
    cache, kv = filled(P, torch, batch, 2, 64)
    q = f16(np.random.default_rng(2), 3, 2, 64)
    want, tol = attention64(q, kv, batch, 0.125, max_q=max_q)
    for starts, rows in (([0, 1, 5, 6], [0]), ([0, 1, 0, 1], None), ([-1, 0, 1, 2], None)):
        st = torch.tensor(starts, dtype=torch.int32, device="cuda")
        out = torch.full((3, 2, 64), 3.0, dtype=torch.float16, device="cuda")
        got = cache.attention(torch.from_numpy(q).cuda(), *batch.args[:2], st, max_q, out=out).cpu().numpy()
        if rows:
            check(got, want, tol, [r for r in batch.rows() if r[0] in rows])
        untouched = [t for t in range(3) if not any(0 <= starts[b] <= t < starts[b + 1] <= 3 for b in range(3))]
        assert (got[untouched] == 3).all()


@pytest.mark.parametrize("new", [1, 20])
def test_a_captured_step_follows_the_batch(P, torch, new):
    """Append and attention captured once, replayed with other lengths, pages and rows; two graphs at once on two streams, workspaces of their own."""
    rng = np.random.default_rng(11)
    h_q, h_kv, d, B = 8, 2, 128, 3
    lens = [[30, 25, 20], [31, 26, 200], [200, 27, 21]]
    big = Batch(torch, [256] * B, [new] * B, 16)
    cos, sin = P.qlinear_rope_tables(256, d, device="cuda")
    caches = [P.PagedKV(big.n_pages, 16, h_kv, d) for _ in range(2)]
    hist = torch.from_numpy(f16(rng, 3 * 256, h_kv, d)).cuda()
    q, k, v = (torch.zeros((B * new, h, d), dtype=torch.float16, device="cuda") for h in (h_q, h_kv, h_kv))
    table, kv_len, q_start = big.args[0].clone(), big.args[1].clone(), big.args[2]

    def step(c):
        turned = c.append(k, v, table, kv_len, q_start, q=q, cos=cos, sin=sin)
        return c.attention(turned, table, kv_len, q_start, new)
    step(caches[0]), step(caches[1])
    for c in caches:
        c.append(hist, hist.flip(0), *big.whole)
    graphs, outs = [], []
    for c in caches:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(c))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for n, ls in enumerate(lens):
        kv_len.copy_(torch.tensor(ls, dtype=torch.int32))
        table.copy_(big.args[0][torch.randperm(B, generator=torch.Generator().manual_seed(n))].clone())
        for t in (q, k, v):
            t.copy_(torch.from_numpy(f16(rng, *t.shape)))
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and outs[0].any()
        eager = P.PagedKV(big.n_pages, 16, h_kv, d)
        eager.pool.copy_(caches[0].pool)
        assert torch.equal(step(eager), outs[0])


@pytest.mark.parametrize("new", [1, 50])
def test_another_stream_and_determinism(P, torch, new):
    batch = Batch(torch, [3000, 60, 999], [new] * 3, 16)
    cache, kv = filled(P, torch, batch, 4, 64)
    q = torch.from_numpy(f16(np.random.default_rng(5), batch.T, 8, 64)).cuda()
    torch.cuda.synchronize()
    first = cache.attention(q, *batch.args, new)
    s = torch.cuda.Stream()
    outs = [cache.attention(q, *batch.args, new, stream=s) for _ in range(20)]
    with torch.cuda.stream(s):
        outs.append(cache.attention(q, *batch.args, new))
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


@pytest.mark.parametrize("h_q,h_kv,d", [(32, 8, 128), (16, 8, 64), (8, 4, 256)])
@pytest.mark.parametrize("lens,new", [([3300, 2900, 2501], 3300), ([9001], 400), ([4100] * 24, 1), ([30011, 7], 1)])
def test_long_batches(P, torch, lens, new, h_q, h_kv, d):
    """Enough segments and steps to keep every ring full on every SM: the same bits from every run, and sampled rows against 64 bits."""
    batch = Batch(torch, lens, [new] * len(lens), 64)
    cache, kv = filled(P, torch, batch, h_kv, d)
    q = f16(np.random.default_rng(5), batch.T, h_q, d)
    dev = torch.from_numpy(q).cuda()
    outs = [cache.attention(dev, *batch.args, batch.max_q) for _ in range(8)]
    assert all(torch.equal(outs[0], o) for o in outs)
    rows = batch.rows()
    rows = [rows[i] for i in np.random.default_rng(6).permutation(len(rows))[:24]]
    want, tol = attention64(q, kv, batch, d ** -0.5, rows=rows)
    check(outs[0].cpu().numpy(), want, tol, rows)


@pytest.mark.parametrize("d,new", [(64, 24), (64, 25), (128, 16), (128, 17), (256, 12), (256, 13)])
def test_rows_where_the_kernels_change(P, torch, d, new):
    """The most rows (two query heads a KV head) that the kernel of few rows takes, and one token more."""
    batch = Batch(torch, [300, new, 77], [new] * 3, 16)
    cache, kv = filled(P, torch, batch, 2, d)
    q = f16(np.random.default_rng(8), batch.T, 4, d)
    got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, new).cpu().numpy()
    want, tol = attention64(q, kv, batch, d ** -0.5)
    check(got, want, tol, batch.rows())


def test_two_streams_at_once(P, torch):
    """Prompts and generated tokens of two caches, captured apart and replayed side by side: what each gives alone."""
    jobs = []
    for lens, new, h_kv, d, seed in (([2000, 1500], 2000, 4, 128, 1), ([5000] * 12, 1, 4, 128, 2)):
        batch = Batch(torch, lens, [new] * len(lens), 16, seed=seed)
        cache, _ = filled(P, torch, batch, h_kv, d, seed=seed)
        q = torch.from_numpy(f16(np.random.default_rng(seed), batch.T, 8, d)).cuda()
        jobs.append((cache, q, batch))
    alone = [c.attention(q, *b.args, b.max_q) for c, q, b in jobs]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in jobs]
    for c, q, b in jobs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append([c.attention(q, *b.args, b.max_q) for _ in range(3)])
        graphs.append(g)
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for got, want in zip(outs, alone) for o in got)


def test_many_sequences(P, torch):
    """More sequences than a CTA has threads; most of them short."""
    rng = np.random.default_rng(13)
    lens = [int(x) for x in rng.integers(0, 40, 700)]
    batch = Batch(torch, lens, [1] * 700, 16)
    cache, kv = filled(P, torch, batch, 1, 64)
    q = f16(rng, batch.T, 2, 64)
    got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, 1).cpu().numpy()
    want, tol = attention64(q, kv, batch, 0.125)
    check(got, want, tol, batch.rows())


def test_a_pool_beyond_32_bits(P, torch):
    """Pages whose bytes lie beyond 2^32 of the pool's start."""
    h_kv, d, page = 8, 256, 1024
    n_pages = 1900                                                       # 1024 tokens of 8 heads of 256: 2.36 MB a page
    cache = P.PagedKV(n_pages, page, h_kv, d)
    assert cache.pool.numel() > 2 ** 32
    rng = np.random.default_rng(1)
    k, v = f16(rng, 300, h_kv, d), f16(rng, 300, h_kv, d)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = i32([[n_pages - 1]])
    cache.append(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), table, i32([300]), i32([0, 300]))
    got_k, got_v = cache.read(table, i32([300]), i32([0, 300]), 300)
    assert (got_k.cpu().numpy() == held(k).astype(np.float16)).all() and (got_v.cpu().numpy() == held(v).astype(np.float16)).all()
    assert not cache.pool[: n_pages - 1].any()
    for new in (1, 40):
        batch = Batch(torch, [300], [new], page)
        q = f16(rng, new, 8, d)
        got = cache.attention(torch.from_numpy(q).cuda(), table, i32([300]), i32([0, new]), new).cpu().numpy()
        want, tol = attention64(q, [(held(k), held(v))], batch, d ** -0.5)
        check(got, want, tol, batch.rows())


def test_refusals(P, torch):
    batch = Batch(torch, [20, 20], [1, 1], 16)
    cache, _ = filled(P, torch, batch, 2, 64)
    z = lambda *s, **k: torch.zeros(s, dtype=k.get("dtype", torch.float16), device=k.get("device", "cuda"))
    table, kv_len, q_start = batch.args
    good = (z(2, 4, 64), *batch.args, 1)
    cache.attention(*good)

    def refused(call, status=P.QL_ERR_INVALID_ARG):
        with pytest.raises(P.QLinearError) as e:
            call()
        assert e.value.status == status
    for q in (z(2, 3, 64), z(2, 4, 32), z(2, 4, 64, dtype=torch.float32), z(2, 4, 64, device="cpu"), z(2, 64, 4).transpose(1, 2), z(2, 4 * 64 + 1)[:, 1:], z(2, 0, 64)):
        refused(lambda: cache.attention(q, *batch.args, 1))
    refused(lambda: cache.attention(z(2 * 4 * 64 + 1)[1:].view(2, 4, 64), *batch.args, 1))               # not 16-byte aligned
    refused(lambda: cache.attention(good[0], table.long(), kv_len, q_start, 1))
    refused(lambda: cache.attention(good[0], table, kv_len[:1], q_start, 1))
    refused(lambda: cache.attention(good[0], table, kv_len, q_start[:2], 1))
    refused(lambda: cache.attention(good[0], table.cpu(), kv_len, q_start, 1))
    refused(lambda: cache.attention(good[0], table, kv_len, q_start, -1))
    refused(lambda: cache.attention(*good, window=-1))
    refused(lambda: cache.attention(*good, softcap=-1.0))
    refused(lambda: cache.attention(*good, scale=float("nan")))
    refused(lambda: cache.attention(*good, out=z(2, 4, 64, dtype=torch.float32)))
    refused(lambda: cache.attention(*good, out=z(3, 4, 64)))
    refused(lambda: cache.attention(*good, out=good[0]))
    k, v, q = z(2, 2, 64), z(2, 2, 64), z(2, 4, 64)
    cos = torch.ones((8, 32), device="cuda")
    cache.append(k, v, *batch.args, q=q, cos=cos, sin=cos)
    refused(lambda: cache.append(z(2, 3, 64), v, *batch.args))
    refused(lambda: cache.append(k, z(3, 2, 64), *batch.args))
    refused(lambda: cache.append(k, v, *batch.args, q=z(3, 4, 64)))
    refused(lambda: cache.append(k, v, *batch.args, cos=cos))
    refused(lambda: cache.append(k, v, *batch.args, cos=cos, sin=cos[:4]))
    refused(lambda: cache.append(k, v, *batch.args, cos=cos[:, :12].contiguous(), sin=cos[:, :12].contiguous()))
    refused(lambda: cache.append(k, v, *batch.args, cos=torch.ones((8, 40), device="cuda"), sin=torch.ones((8, 40), device="cuda")))
    refused(lambda: cache.append(k, v, *batch.args, q_out=q))
    refused(lambda: cache.append(k, v, *batch.args, q=q, q_out=z(2, 8, 64)[:, ::2]))
    refused(lambda: cache.read(*batch.args, -1))
    for args in ((4, 15, 2, 64), (4, 24, 2, 64), (4, 2048, 2, 64), (4, 16, 2, 96), (0, 16, 2, 64), (4, 16, 0, 64)):
        refused(lambda: P.PagedKV(*args), P.QL_ERR_UNSUPPORTED)
    cache.close()
    refused(lambda: cache.attention(*good))
    refused(lambda: cache.append(k, v, *batch.args))
    refused(lambda: cache.read(*batch.args, 2))


@pytest.mark.parametrize("max_q,width,taken", [(1, 1 << 19, True), (1, 1 << 20, False), (64, 1 << 21, True), (64, 1 << 22, False)])
def test_work_that_32_bits_do_not_count(P, torch, max_q, width, taken):
    """2048 sequences whose table has room for `width` pages of 16 tokens and no page in it: the steps of a KV head are width + 33 a sequence, width / 4 + 9 with
    many rows.  No sequence has a token or a row, so none of the table is read (it is shorter than it says)."""
    B = 2048
    cache = P.PagedKV(1, 16, 1, 64)
    kv_len, q_start = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    q = torch.zeros((2, 1, 64), dtype=torch.float16, device="cuda")
    need = P.binding.lib.qlinear_paged_attention_workspace(cache._h, 1, B, max_q)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7)
    table = torch.full((1 << 10,), -1, dtype=torch.int32, device="cuda")
    status = P.binding.lib.qlinear_paged_attention(cache._h, q.data_ptr(), 64, out.data_ptr(), 64, 1, table.data_ptr(), width, width, kv_len.data_ptr(), q_start.data_ptr(), B, 2,
                                                   max_q, 1.0, 0.0, 0, work.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == (P.binding.QL_OK if taken else P.QL_ERR_INVALID_ARG) and (out == 7).all()


def test_empty_calls(P, torch):
    batch = Batch(torch, [20], [1], 16)
    cache, _ = filled(P, torch, batch, 2, 64)
    z = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    none = (torch.zeros((0, 1), dtype=torch.int32, device="cuda"), i32(), i32(0))
    before = cache.pool.clone()
    assert cache.attention(z(0, 4, 64), *none, 0).shape == (0, 4, 64)
    assert cache.append(z(0, 2, 64), z(0, 2, 64), *none, q=z(0, 4, 64)).shape == (0, 4, 64) and cache.append(z(0, 2, 64), z(0, 2, 64), *none) is None
    assert cache.read(*none, 0)[0].shape == (0, 2, 64)
    cache.append(z(3, 2, 64) + 1, z(3, 2, 64), *none)                    # rows of no sequence
    assert torch.equal(before, cache.pool)


def test_both_halves_agree(P, torch, monkeypatch):
    batch = Batch(torch, [40, 300], [3, 3], 16)
    q, k, v = (torch.from_numpy(f16(np.random.default_rng(5), 6, h, 128)).cuda() for h in (8, 2, 2))
    cos, sin = P.qlinear_rope_tables(512, 64, device="cuda")

    def calls():
        cache, _ = filled(P, torch, batch, 2, 128)
        o, a = torch.zeros_like(q), torch.zeros_like(q)
        assert cache.append(k, v, *batch.args, q=q, cos=cos, sin=sin, interleaved=True, q_out=o) is o and cache.append(k, v, *batch.args) is None
        assert cache.attention(o, *batch.args, 3, out=a) is a
        return [o, a, cache.attention(o, *batch.args, 3, scale=1, softcap=9, window=30), cache.append(k.view(6, -1), v.view(6, -1), *batch.args, q=q.view(6, -1)), *cache.read(*batch.args, 6), cache.pool]
    native, taken = P.binding._serving, []

    class Recorded:
        def __getattr__(self, name):
            def call(*a):
                taken.append(getattr(native, name)(*a))
                return taken[-1]
            return call

    class Python:
        def __getattr__(self, name):
            return lambda *a: None
    monkeypatch.setattr(P.binding, "_serving", Recorded())
    fast = calls()
    assert taken and all(t is not None for t in taken)
    monkeypatch.setattr(P.binding, "_serving", Python())
    slow = calls()
    assert all(torch.equal(a, b) and a.shape == b.shape for a, b in zip(fast, slow))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,n,new,h_kv,group", [(400, 8191, 1, 1, 2), (1, 70000, 2500, 4, 8)])
def test_many_light_tokens_behind_a_heavy_one(P, torch, B, n, new, h_kv, group, d):
    """The first token has nearly all the weight and no value, every other one 2^-25.6 of that weight: the result is what the light ones add up to.  Bound: the scores' sums (and, with
    many rows, the keys' rounding), weights, values and result in fp16 (2^-11 each), and 2^-32 of the largest weight for every light one: half a step of fp16 below 2^-14, where weights up to 2^7 are held."""
    cache = P.PagedKV(-(-n // 16), 16, h_kv, d)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = torch.arange(-(-n // 16), dtype=torch.int32, device="cuda").expand(B, -1).contiguous()           # (all sequences are the same tokens)
    k, v = (torch.zeros((n, h_kv, d), dtype=torch.float16, device="cuda") for _ in range(2))
    k[0], v[1:] = 1, 1
    cache.append(k, v, table[:1], i32([n]), i32([0, n]))
    one = held(np.ones((1, d), np.float16))[0]
    scale = 25.6 * np.log(2) / one.sum()
    q = torch.ones((B * new, h_kv * group, d), dtype=torch.float16, device="cuda")
    got = cache.attention(q, table, i32([n] * B), i32((np.arange(B + 1) * new).tolist()), new, scale=scale).double().cpu().numpy()
    x0 = one.sum() * float(np.float32(scale))
    light, w = n - new + np.tile(np.arange(new), B), np.exp(-x0)
    y = light * w / (1 + light * w) * one[0]
    dx = ((d + 60) * 2.0 ** -24 + (2.0 ** -11 if new > 1 else 0)) * x0
    tol = y * (2 * np.expm1(dx) + 3 * 2.0 ** -11 + n * 2.0 ** -24) + 2.0 ** -32 * light / (1 + light * w) + 2.0 ** -25
    assert (np.abs(got - y[:, None, None]).max((1, 2)) <= tol).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("softcap", [1e-3, 128.0, 1e3, 1e5, 1e8, 3e38])
def test_soft_caps_of_every_size(P, torch, softcap, new, d):
    """Caps far below the scores and far above them, where capped scores are the scores.  Up to 128 a score is off by roundings of numbers up to the cap (as in attention64); above, by those of the score
    alone: exponential form for |y| >= 1/4, 1.5 * 2^-22 absolute of tanh(y) >= 0.244 (2 ulp of the exponential, 1 of the reciprocal, a sum, a product) and 3 roundings of its argument, and 2 of the factor, 30 * 2^-24 in all;
    series below, 6 * 2^-24 cut off and 8 roundings."""
    batch = Batch(torch, [500, 61], [new, new], 16)
    cache, kv = filled(P, torch, batch, 2, d)
    q = f16(np.random.default_rng(3), batch.T, 4, d)
    key = 2.0 ** -11 if new * 2 > {64: 48, 128: 32, 256: 24}[d] else 0.0
    for size in (1.0, 300.0):                                            # (scores of a few units; of hundreds: tanh of 1e3 on both sides of 1/4)
        scale = size * d ** -0.5
        got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, new, scale=scale, softcap=softcap).cpu().numpy().astype(np.float64)
        for t, b, pos in batch.rows():
            for h in range(4):
                k, v, q64 = kv[b][0][:pos + 1, h // 2], kv[b][1][:pos + 1, h // 2], q[t, h].astype(np.float64)
                x = softcap * np.tanh(k @ q64 * scale / softcap)
                dx = np.minimum((key + (d + 40) * 2.0 ** -24) * (np.abs(k) @ np.abs(q64)) * scale, 2 * softcap) + (16 * 2.0 ** -24 * softcap if softcap <= 128 else 40 * 2.0 ** -24 * np.abs(x))
                w = np.exp(x - x.max())
                rel = np.expm1(dx + 2.0 ** -21 * (1 + np.abs(x - x.max()))).max()
                want = w @ v / w.sum()
                tol = (2 * rel + 2 * 2.0 ** -11 + len(k) * 2.0 ** -24) * (w @ np.abs(v)) / w.sum() + 2.0 ** -32 / w.sum() * np.abs(v).sum(0)
                assert (np.abs(got[t, h] - want) <= 1.01 * tol + 2.0 ** -11 * np.abs(want) + 2.0 ** -25).all(), (t, h, size)


@pytest.mark.parametrize("new,most", [(1, 1), (3, 3), (3, 2), (70, 70), (700, 700), (700, 300)])
@pytest.mark.parametrize("window", [0, 90])
def test_a_table_that_ends_with_the_last_token(P, torch, new, most, window):
    """A table said to be wide that holds the entries up to the last row's token (or to that of the last row served) and no more: none behind them is read."""
    n, d = 1111, 128
    batch = Batch(torch, [n], [new], 16)
    cache, _ = filled(P, torch, batch, 2, d)
    q = torch.from_numpy(f16(np.random.default_rng(4), new, 8, d)).cuda()
    want = cache.attention(q, *batch.args, most, window=window, out=torch.zeros_like(q))
    short = batch.args[0][0, :-(-(n - new + most) // 16)].clone()
    work = torch.empty(P.lib.qlinear_paged_attention_workspace(cache._h, 8, 1, most), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    assert P.lib.qlinear_paged_attention(cache._h, q.data_ptr(), 8 * d, out.data_ptr(), 8 * d, 8, short.data_ptr(), 1 << 20, 1 << 20, batch.args[1].data_ptr(), batch.args[2].data_ptr(), 1, new, most,
                                         d ** -0.5, 0.0, window, work.data_ptr(), work.numel(), torch.cuda.current_stream().cuda_stream) == P.binding.QL_OK
    assert torch.equal(out, want)


def test_numbers_beyond_32_bits(P, torch):
    """Refused: their lower 32 bits would be another call (a window of 5, a single row)."""
    batch = Batch(torch, [60], [2], 16)
    cache, _ = filled(P, torch, batch, 2, 64)
    q = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda")
    for call in (lambda: cache.attention(q, *batch.args, 2, window=2 ** 32 + 5), lambda: cache.attention(q, *batch.args, 2 ** 32 + 1), lambda: cache.read(*batch.args, 2 ** 32)):
        with pytest.raises(P.QLinearError) as e:
            call()
        assert e.value.status == P.QL_ERR_INVALID_ARG
    cache.attention(q, *batch.args, 2, window=2 ** 31 - 1)


@pytest.mark.parametrize("new", [1, 40])
def test_the_largest_scale(P, torch, new):
    """Scores of -2e29 are scores (all the same here, so the result is the values' mean, half a step of fp16 each for a value, the weights and the result); scales that would let them pass -1e30 are refused."""
    batch = Batch(torch, [60], [new], 16)
    cache = P.PagedKV(batch.n_pages, 16, 2, 256)
    x = torch.full((60, 2, 256), 1000.0, dtype=torch.float16, device="cuda")
    cache.append(x, x, *batch.whole)
    q = torch.full((new, 4, 256), -1000.0, dtype=torch.float16, device="cuda")
    for scale in (1e15, 1e12):
        out = cache.attention(q, *batch.args, new, scale=scale).double()
        want = held(x[:1, :1].cpu().numpy()).flat[0]
        assert ((out - want).abs() <= 3 * 2.0 ** -11 * want).all()
    for scale in (1.1e15, -1e16, 1e30, -3e38, float("inf"), float("nan")):
        with pytest.raises(P.QLinearError) as e:
            cache.attention(q, *batch.args, new, scale=scale)
        assert e.value.status == P.QL_ERR_INVALID_ARG


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("exponent", [20, 24, 26, 27, 28, 29, 32])
def test_scores_of_millions(P, torch, new, exponent):
    """Scores that are far apart: the heaviest token takes all, or shares with those that are the same.  Tokens 5 and 50 and, for 60, the same key; the others' scores lie 2^-6 of that score below, many powers of two."""
    batch = Batch(torch, [61], [new], 16)
    cache = P.PagedKV(batch.n_pages, 16, 2, 64)
    k = torch.full((61, 2, 64), 7.0, dtype=torch.float16, device="cuda")             # (held exactly: 7 times a scale of 1)
    k[:, :, 1] = 0
    k[[5, 50, 60], :, 1] = 1                                             # (a power of 2^exponent / 63 more for each of these)
    v = torch.from_numpy(f16(np.random.default_rng(2), 61, 2, 64)).cuda()
    cache.append(k, v, *batch.whole)
    q = torch.ones((new, 4, 64), dtype=torch.float16, device="cuda")
    scale = 2.0 ** exponent / (63 * 7) * np.log(2)
    out = cache.attention(q, *batch.args, new, scale=scale).double().cpu().numpy()
    values = held(v.cpu().numpy())
    for i in range(new):
        see = [t for t in (5, 50, 60) if t <= 61 - new + i]
        want = values[see].mean(0).repeat(2, 0)
        assert (np.abs(out[i] - want) <= 2 * 2.0 ** -11 * np.abs(values[see]).mean(0).repeat(2, 0) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25).all()


@pytest.mark.parametrize("h_q,h_kv,d,new", [(32, 8, 64, 13), (32, 8, 128, 9), (16, 8, 256, 13)])
def test_more_segments_than_a_round_takes(P, torch, h_q, h_kv, d, new):
    """The most sequences a call takes, short, with rows enough for the kernel of many rows: about 110 segments a CTA, which lists 64 at a time.  The same bits from every run, sampled rows against 64 bits."""
    rng = np.random.default_rng(d)
    lens = [int(x) for x in rng.integers(0, 90, 2048)]
    batch = Batch(torch, lens, [new] * 2048, 16, behind=1)
    assert sum(n > 0 for n in lens) * h_kv > 2 * 64 * torch.cuda.get_device_properties(0).multi_processor_count * 0.8
    cache, kv = filled(P, torch, batch, h_kv, d)
    q = f16(rng, batch.T, h_q, d)
    dev = torch.from_numpy(q).cuda()
    outs = [cache.attention(dev, *batch.args, new, out=torch.full_like(dev, 9)) for _ in range(4)]
    assert all(torch.equal(outs[0], o) for o in outs) and (outs[0][-1] == 9).all()
    rows = batch.rows()
    rows = [rows[i] for i in rng.permutation(len(rows))[:200]]
    want, tol = attention64(q, kv, batch, d ** -0.5, rows=rows)
    check(outs[0].cpu().numpy(), want, tol, rows)


@pytest.mark.parametrize("h_q,h_kv,d", [(32, 8, 128), (8, 4, 256), (14, 2, 64)])
@pytest.mark.parametrize("new", [[1, 400, 3, 1, 0, 2], [1, 4, 2, 6, 1, 3]])
@pytest.mark.parametrize("window", [0, 1000])
def test_rows_of_every_kind_in_one_call(P, torch, h_q, h_kv, d, new, window):
    """A prompt's chunk beside generated tokens over thousands of cached ones, and a few tokens of each sequence, by the kernel that the largest number of rows asks for."""
    lens = [3000, 4100, 2500, 5, 40, 1999]
    batch = Batch(torch, lens, new, 32, seed=3, before=1, behind=2)
    cache, kv = filled(P, torch, batch, h_kv, d)
    q = f16(np.random.default_rng(8), batch.T, h_q, d)
    out = torch.full((batch.T, h_q, d), 9.0, dtype=torch.float16, device="cuda")
    got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, batch.max_q, window=window, out=out).cpu().numpy()
    rows = [r for r in batch.rows() if batch.new[r[1]] < 10 or r[0] % 23 == 0]
    want, tol = attention64(q, kv, batch, d ** -0.5, 0.0, window, rows=rows)
    check(got, want, tol, rows)
    assert (got[0] == 9).all() and (got[-2:] == 9).all()


@pytest.mark.parametrize("h_kv,d", [(2, 64), (2, 128), (2, 256)])
def test_the_most_sequences(P, torch, h_kv, d):
    """2048 sequences of a token each: the plan of the batch at its largest, in the kernel of few rows."""
    rng = np.random.default_rng(d)
    lens = [int(x) for x in rng.integers(0, 200, 2048)]
    batch = Batch(torch, lens, [1] * 2048, 16)
    cache, kv = filled(P, torch, batch, h_kv, d)
    q = f16(rng, batch.T, 4, d)
    got = cache.attention(torch.from_numpy(q).cuda(), *batch.args, 1).cpu().numpy()
    rows = [r for r in batch.rows() if r[1] % 7 == 0]
    want, tol = attention64(q, kv, batch, d ** -0.5, rows=rows)
    check(got, want, tol, rows)


@pytest.mark.parametrize("new", [1, 50])
def test_a_table_cut_from_a_wider_one(P, torch, new):
    batch = Batch(torch, [300, 170, 44], [new] * 3, 16)
    k, v = (torch.from_numpy(f16(np.random.default_rng(s), batch.T, 2, 128)).cuda() for s in (1, 2))
    q = torch.from_numpy(f16(np.random.default_rng(3), batch.T, 8, 128)).cuda()
    wide = torch.full((3, batch.table.shape[1] + 9), 2 ** 30, dtype=torch.int32, device="cuda")
    wide[:, 4:-5] = batch.args[0]
    results = []
    for table in (batch.args[0], wide[:, 4:-5]):
        cache, _ = filled(P, torch, batch, 2, 128)
        cache.append(k, v, table, *batch.args[1:])
        results.append([cache.pool, *cache.read(table, *batch.args[1:], batch.T), cache.attention(q, table, *batch.args[1:], new)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_the_ctas_of_a_call_run_at_once(P, torch, d):
    """The kernel of few rows cuts its work into spans of equal length for CTAs that run side by side: as many as fit, by the runtime's own count, up to two an SM, whatever the number of sequences."""
    import ctypes
    cache, fit = P.PagedKV(1, 16, 1, d), ctypes.c_int32()
    launched = []
    for B in (1, 24, 700, 1500, *range(1600, 1720, 4), 2048):
        launched.append(P.lib.qlinear_debug_paged_ctas(cache._h, B, ctypes.byref(fit)))
        assert launched[-1] == min(fit.value, 2) > 0, (B, launched[-1], fit.value)
    assert set(launched) == {64: {2}, 128: {1, 2}, 256: {1}}[d]
    assert P.lib.qlinear_debug_paged_ctas(None, 1, ctypes.byref(fit)) == 0 == P.lib.qlinear_debug_paged_ctas(cache._h, 2049, ctypes.byref(fit))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_workspace_for_the_most_sequences_serves_fewer(P, torch, d):
    batch = Batch(torch, [100, 7], [1, 1], 16)
    cache, _ = filled(P, torch, batch, 2, d)
    q = torch.from_numpy(f16(np.random.default_rng(4), 2, 4, d)).cuda()
    work = torch.empty(P.lib.qlinear_paged_attention_workspace(cache._h, 4, 2048, 1), dtype=torch.uint8, device="cuda")
    out, table = torch.zeros_like(q), batch.args[0]
    assert P.lib.qlinear_paged_attention(cache._h, q.data_ptr(), 4 * d, out.data_ptr(), 4 * d, 4, table.data_ptr(), table.stride(0), table.shape[1], batch.args[1].data_ptr(), batch.args[2].data_ptr(), 2, 2, 1,
                                         d ** -0.5, 0.0, 0, work.data_ptr(), work.numel(), torch.cuda.current_stream().cuda_stream) == P.binding.QL_OK
    assert torch.equal(out, cache.attention(q, *batch.args, 1)) and out.any()


@pytest.mark.parametrize("n", [0, -1, -7, -2 ** 31, -2 ** 31 + 3])
def test_lengths_below_the_rows(P, torch, n):
    """Rows of a sequence said to be shorter than they are many lie before its first token: left by append, zeros from attention (the rows served), whatever the length."""
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    batch = i32(0, 1)[None], i32(n), i32(0, 8)
    cache = P.PagedKV(2, 16, 2, 64)
    k, q = (torch.ones((8, h, 64), dtype=torch.float16, device="cuda") for h in (2, 4))
    cos, sin = P.qlinear_rope_tables(32, 64)
    mark = torch.full_like(q, 7)
    cache.append(k, k, *batch, q=q, cos=cos, sin=sin, q_out=mark)
    assert (mark == 7).all() and not cache.pool.any()
    for most in (8, 3):
        out = cache.attention(q, *batch, most, out=torch.full_like(q, 7))
        assert not out[:most].any() and (out[most:] == 7).all()
    many = torch.ones((60, 4, 64), dtype=torch.float16, device="cuda")
    assert not cache.attention(many, *batch[:2], i32(0, 60), 60).any()
