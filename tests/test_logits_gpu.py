"""Penalties, biases and masks on logits against a plain implementation (numpy, 64 bits)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P(_built_library):
    import paper_2505_00232_b200 as P
    return P


def adjusted(x, tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, mask):
    """(result in 64 bits, bound of the fp32 steps)"""
    y = x.astype(np.float64)
    R, V = y.shape
    tol = np.zeros_like(y)
    for r in range(R):
        seen, said = np.zeros(V, bool), np.zeros(V)
        if tokens is not None:
            h = tokens[start[r]:start[r + 1]]
            for i, t in enumerate(h):
                if 0 <= t < V:
                    seen[t] = True
                    said[t] += n_prompt is None or i >= n_prompt[r]
        a = np.abs(y[r])
        with np.errstate(invalid="ignore"):
            y[r, seen] = np.where(y[r, seen] > 0, y[r, seen] / rep[r], y[r, seen] * rep[r])
            a = np.maximum(a, np.abs(y[r]))
            y[r] -= np.where(said > 0, freq[r] * said + pres[r], 0)
        a += np.where(said > 0, abs(freq[r]) * said + abs(pres[r]), 0)
        if ids is not None:
            last = {int(t): v for t, v in zip(ids[b_start[r]:b_start[r + 1]], values[b_start[r]:b_start[r + 1]]) if 0 <= t < V}
            for t, v in last.items():
                y[r, t] += v
                a[t] += abs(v)
        if mask is not None:
            off = (mask[r, np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1 == 0
            y[r, off] = -np.inf
        tol[r] = np.where(np.isfinite(a), 4 * 2.0 ** -24 * a, 0)         # four rounded fp32 operations on numbers up to a
    return y, tol


def check(got, want, tol, dtype):
    got = got.astype(np.float64)
    eps = 2.0 ** -11 if dtype == np.float16 else 2.0 ** -24
    fine = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all() and (got[~fine & ~np.isnan(want)] == want[~fine & ~np.isnan(want)]).all()
    assert (np.abs(got - want)[fine] <= (tol + eps * (np.abs(want) + tol) + 2.0 ** -25)[fine]).all()


def inputs(rng, R, V, n, dtype):
    x = (3 * rng.standard_normal((R, V))).astype(dtype)
    lens = rng.integers(0, n + 1, R)
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    tokens = rng.integers(-2, V + 2, start[-1]).astype(np.int32)         # (some outside the vocabulary)
    if len(tokens) > 4:
        tokens[::3] = tokens[0]                                          # one that comes back often
    n_prompt = (lens // 2).astype(np.int32)
    rep, pres, freq = (1 + rng.random(R)).astype(np.float32), rng.random(R).astype(np.float32), rng.random(R).astype(np.float32)
    nb = rng.integers(0, 9, R)
    b_start = np.concatenate([[0], np.cumsum(nb)]).astype(np.int32)
    ids = rng.integers(-1, V + 1, b_start[-1]).astype(np.int32)
    if len(ids) > 3:
        ids[1] = ids[0]                                                  # the same token twice: the last counts
    values = (5 * rng.standard_normal(len(ids))).astype(np.float32)
    mask = rng.integers(0, 2 ** 32, (R, (V + 31) // 32 + 1), dtype=np.uint64).astype(np.uint32)
    return x, tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, mask


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("R,V,n", [(1, 1, 3), (3, 31, 10), (2, 33, 0), (5, 2047, 300), (4, 2049, 300), (1, 50257, 5000), (60, 32001, 40), (40, 70003, 200)])
def test_parity(P, dtype, R, V, n):
    import torch
    a = inputs(np.random.default_rng(V + R), R, V, n, dtype)
    up = lambda t: None if t is None else torch.from_numpy(t.view(np.int32) if t.dtype == np.uint32 else t).cuda()
    dev = [up(t) for t in a]
    want, tol = adjusted(*a)
    x, tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, mask = dev
    got = P.qlinear_adjust_logits(x, tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, mask)
    check(got.cpu().numpy(), want, tol, dtype)
    # in place; a row of the caller's own stride, with another alignment of the result
    y = x.clone()
    assert P.qlinear_adjust_logits(y, tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, mask, out=y) is y and torch.equal(y, got)
    wide, other = torch.zeros((R, V + 9), dtype=x.dtype, device="cuda"), torch.full((R, V + 6), 5.0, dtype=x.dtype, device="cuda")
    wide[:, 1:V + 1] = x
    P.qlinear_adjust_logits(wide[:, 1:V + 1], tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, mask, out=other[:, 4:V + 4])
    assert torch.equal(other[:, 4:V + 4], got) and (other[:, :4] == 5).all() and (other[:, V + 4:] == 5).all()
    # each part alone
    one, none = np.ones(R, np.float32), np.zeros(R, np.float32)
    parts = [(dict(), (None,) * 3 + (one, none, none) + (None,) * 4), (dict(mask=mask), (None,) * 3 + (one, none, none, None, None, None, a[10])),
             (dict(bias_ids=ids, bias_values=values, bias_start=b_start), (None,) * 3 + (one, none, none) + a[7:10] + (None,)),
             (dict(tokens=tokens, start=start, repetition=rep), a[1:3] + (None, a[4], none, none) + (None,) * 4),
             (dict(tokens=tokens, start=start, presence=pres, frequency=freq), a[1:3] + (None, one, a[5], a[6]) + (None,) * 4)]
    for kwargs, plain in parts:
        want, tol = adjusted(a[0], *plain)
        check(P.qlinear_adjust_logits(x, **kwargs).cpu().numpy(), want, tol, dtype)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_what_is_not_finite(P, dtype):
    """Infinities and NaN in masked and in allowed places, biases of minus infinity, a row whose mask leaves nothing."""
    import torch
    V = 100
    x = np.zeros((3, V), dtype)
    x[:, 0], x[:, 1], x[:, 2], x[:, 3] = np.nan, np.inf, -np.inf, np.finfo(dtype).min
    mask = np.zeros((3, 4), np.uint32)
    mask[1] = 0xFFFFFFFF
    mask[2] = 0b1010
    tokens, start = np.array([1, 2, 3, 5, 5] * 3, np.int32), np.array([0, 5, 10, 15], np.int32)
    ids, values, b_start = np.array([7, 8], np.int32), np.array([-np.inf, np.inf], np.float32), np.array([0, 0, 2, 2], np.int32)
    rep, pres, freq = np.full(3, 1.5, np.float32), np.full(3, 0.25, np.float32), np.full(3, 0.5, np.float32)
    up = lambda t: torch.from_numpy(t.view(np.int32) if t.dtype == np.uint32 else t).cuda()
    got = P.qlinear_adjust_logits(up(x), up(tokens), up(start), None, up(rep), up(pres), up(freq), up(ids), up(values), up(b_start), up(mask)).cpu().numpy()
    assert (got[0] == -np.inf).all()
    assert np.isnan(got[1, 0]) and got[1, 1] == np.inf and got[1, 2] == -np.inf and got[1, 7] == -np.inf and got[1, 8] == np.inf and got[1, 5] == -1.25
    allowed = np.isin(np.arange(V) % 32, [1, 3])                         # (of every word)
    assert (got[2, ~allowed] == -np.inf).all() and got[2, 1] == np.inf and (got[2, [33, 35, 65, 67, 97, 99]] == 0).all()


@pytest.mark.parametrize("R", [2, 40])
def test_more_biases_than_count(P, R):
    """The last 65535 biases of a row count, for few rows and for many."""
    import torch
    V, n = 70003, 70000
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    values = torch.rand(n, device="cuda") + 1
    start = torch.full((R + 1,), n, dtype=torch.int32, device="cuda")
    start[:R // 2] = 0                                                   # (one row has them all)
    y = P.qlinear_adjust_logits(torch.zeros((R, V), device="cuda"), bias_ids=ids, bias_values=values, bias_start=start)
    want = torch.zeros((R, V), device="cuda")
    want[R // 2 - 1, n - 65535:n] = values[n - 65535:]
    assert torch.equal(y, want)


def test_capture_streams_and_halves(P, monkeypatch):
    import torch
    a = inputs(np.random.default_rng(3), 7, 5000, 90, np.float16)
    dev = [torch.from_numpy(t.view(np.int32) if t.dtype == np.uint32 else t).cuda() for t in a]
    want = P.qlinear_adjust_logits(*dev)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = P.qlinear_adjust_logits(*dev, stream=s)                        # (Python's half)
    s.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = P.qlinear_adjust_logits(*dev)
    new = inputs(np.random.default_rng(3), 7, 5000, 90, np.float16)
    dev[0].copy_(torch.from_numpy(new[0] * np.float16(-1)))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, P.qlinear_adjust_logits(*dev)) and not torch.equal(y, want)
    native, taken = P.binding._serving, []

    class Recorded:
        def adjust_logits(self, *a):
            taken.append(native.adjust_logits(*a))
            return taken[-1]
    monkeypatch.setattr(P.binding, "_serving", Recorded())
    P.qlinear_adjust_logits(*dev)
    P.qlinear_adjust_logits(dev[0].float()[:, :4000], out=dev[0].float()[:, :4000])
    assert len(taken) == 2 and all(t is not None for t in taken)


def test_refusals(P):
    import torch
    a = inputs(np.random.default_rng(3), 4, 500, 9, np.float16)
    x, tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, mask = [torch.from_numpy(t.view(np.int32) if t.dtype == np.uint32 else t).cuda() for t in a]

    def refused(*args, **kwargs):
        with pytest.raises(P.QLinearError) as e:
            P.qlinear_adjust_logits(*args, **kwargs)
        assert e.value.status == P.QL_ERR_INVALID_ARG
    refused(x.to(torch.bfloat16))
    refused(x.cpu())
    refused(x.t())
    refused(x[0])
    refused(x, tokens=tokens)
    refused(x, tokens=tokens.long(), start=start)
    refused(x, tokens=tokens, start=start[:3])
    refused(x, tokens=tokens, start=start, n_prompt=n_prompt[:2])
    refused(x, repetition=rep.double())
    refused(x, bias_ids=ids, bias_values=values)
    refused(x, bias_ids=ids, bias_values=values[:-1], bias_start=b_start)
    refused(x, mask=mask[:, :15].contiguous())
    refused(x, mask=mask[:3])
    refused(x, out=x.float())
    refused(x, out=x[:, :499])


def test_the_largest_vocabulary(P):
    """2^31 - 1 tokens of a row: the first and the last ones, and the bits of the last word of the mask."""
    import torch
    V = 2 ** 31 - 1
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    x = torch.zeros((1, V), dtype=torch.float16, device="cuda")
    at = torch.tensor([0, 3, 2 ** 30, V - 2050, V - 2, V - 1], device="cuda")
    history = dict(tokens=i32(3, V - 1, -1, -2 ** 31), start=i32(0, 4), presence=torch.ones(1, device="cuda"))
    biases = dict(bias_ids=i32(3, V - 2, 2 ** 30), bias_values=torch.tensor([5.0, 6.0, 7.0], device="cuda"), bias_start=i32(0, 3))
    y = P.qlinear_adjust_logits(x, **history, **biases)
    assert y[0, at].tolist() == [0, 4, 7, 0, 6, -1] and int(y.count_nonzero()) == 4
    mask = torch.full((1, 2 ** 26), -1, dtype=torch.int32, device="cuda")
    mask[0, 0], mask[0, -1] = ~1, ~(1 << 30)
    y = P.qlinear_adjust_logits(x, **history, **biases, mask=mask, out=y)
    assert y[0, at].tolist() == [-float("inf"), 4, 7, 0, 6, -float("inf")] and int(y.isinf().sum()) == 2
    assert P.qlinear_adjust_logits(x, mask=mask, out=x) is x and x[0, at].tolist() == [-float("inf"), 0, 0, 0, 0, -float("inf")]


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("R,V,n", [(16, 256000, 3000), (12, 131072 + 5, 700), (12, 131072, 700)])
def test_vocabularies_of_more_than_one_piece(P, dtype, R, V, n):
    """Many rows, whose seen tokens are adjusted by a CTA per 131072 tokens: history, biases and mask in every piece, and at its ends."""
    import torch
    a = list(inputs(np.random.default_rng(V), R, V, n, dtype))
    ends = np.array([0, 131071, min(131072, V - 1), V - 1], np.int32)
    for r in range(R):
        if a[2][r + 1] - a[2][r] >= 8:
            a[1][a[2][r]:a[2][r] + 4] = a[1][a[2][r + 1] - 4:a[2][r + 1]] = ends
        if a[9][r + 1] - a[9][r] >= 4:
            a[7][a[9][r]:a[9][r] + 4] = ends
    dev = [torch.from_numpy(t.view(np.int32) if t.dtype == np.uint32 else t).cuda() for t in a]
    for masked in (True, False):
        want, tol = adjusted(*a[:10], a[10] if masked else None)
        got = P.qlinear_adjust_logits(*dev[:10], mask=dev[10] if masked else None)
        check(got.cpu().numpy(), want, tol, dtype)
