"""Rotary angle tables against the definition in 64 bits, every scaling."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P(_built_library):
    import paper_2505_00232_b200 as P
    return P


def frequencies(rot, base, scaling, factor, original=8192, slow=1.0, fast=4.0):
    f = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base
        x = b ** (-2 * i / rot)
        if scaling == "linear":
            x /= factor
        elif scaling == "llama3":
            length = 2 * math.pi / x
            if length > original / slow:
                x /= factor
            elif length >= original / fast:
                s = (original / length - slow) / (fast - slow)
                x = (1 - s) * x / factor + s * x
        elif scaling == "yarn":
            at = lambda turns: rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
            low, high = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), rot - 1)
            r = min(max((i - low) / max(high - low, 0.001), 0), 1)
            x = x / factor * r + x * (1 - r)
        f.append(x)
    return np.array(f)


@pytest.mark.parametrize("scaling,turns", [(None, None), ("linear", None), ("ntk", None), ("llama3", (1.0, 4.0)), ("yarn", (1.0, 32.0)), ("llama3", (0.5, 2.0))])
@pytest.mark.parametrize("n_pos,rot,base,first", [(1, 16, 10000.0, 0), (777, 128, 500000.0, 5), (33, 48, 10000.0, 131000), (2, 512, 10000.0, 2 ** 31 - 3), (5000, 64, 10000.0, 0)])
def test_tables(P, scaling, turns, n_pos, rot, base, first):
    """The angle in turns is off by position * 2^-53 of a turn and a few ulp of the frequency (itself good to 8 * 2^-53 relative), its fraction is rounded
    to fp32 (2^-25 of a turn at most), cos and sin to 2 ulp: absolute errors, on numbers up to the magnitude."""
    factor = 8.0
    slow, fast = turns or (None, None)
    cos, sin = P.qlinear_rope_tables(n_pos, rot, base, scaling=scaling, factor=factor, slow=slow, fast=fast, first=first)
    f = frequencies(rot, base, scaling, factor, slow=slow or 1.0, fast=fast or 4.0)
    pos = np.arange(first, first + n_pos, dtype=np.float64)
    angle = np.outer(pos, f)
    m = 0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0
    tol = m * (angle * 32 * 2.0 ** -53 + 2 * math.pi * 2.0 ** -25 + 4 * 2.0 ** -24)
    assert cos.shape == sin.shape == (n_pos, rot // 2)
    assert (np.abs(cos.cpu().numpy() - m * np.cos(angle)) <= tol).all() and (np.abs(sin.cpu().numpy() - m * np.sin(angle)) <= tol).all()


def test_as_the_rotation_takes_them(P):
    """The rotation that reads the tables, against the complex product in 64 bits."""
    import torch
    cos, sin = P.qlinear_rope_tables(40, 64, device="cuda")
    rng = np.random.default_rng(0)
    q, k = (torch.from_numpy(rng.standard_normal((40, h * 64)).astype(np.float16)).cuda() for h in (4, 2))
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    qo = P.qlinear_rope_qkv(q, k, k, pos, cos, sin, 1, 40, 4, 2, 64)[0].cpu().numpy().astype(np.float64)      # [2, 80, 64]
    x = q.cpu().numpy().astype(np.float64).reshape(40, 2, 2, 64)
    z = (x[..., :32] + 1j * x[..., 32:]) * np.exp(1j * np.outer(np.arange(40), 10000.0 ** (-np.arange(32) / 32)))[:, None, None]
    want = np.concatenate([z.real, z.imag], -1).transpose(1, 0, 2, 3).reshape(2, 80, 64)
    assert np.abs(qo - want).max() <= 2.0 ** -10 * np.abs(want).max()


def test_another_stream(P):
    import torch
    s = torch.cuda.Stream()
    a = P.qlinear_rope_tables(3000, 128, stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, P.qlinear_rope_tables(3000, 128)))
    assert P.qlinear_rope_tables(0, 64)[0].shape == (0, 32)


def test_every_position(P):
    """2^31 - 1 positions of the smallest head: the first, some in between and the last ones (bounds: test_tables)."""
    import torch
    torch.cuda.empty_cache()
    n, rot = 2 ** 31 - 1, 16
    if torch.cuda.mem_get_info()[0] < 4 * n * rot + (4 << 30):
        pytest.skip("the tables take 137 GB")
    tables = P.qlinear_rope_tables(n, rot)
    f = frequencies(rot, 10000.0, None, 1.0)
    for pos in (np.arange(300), 2 ** 28 * np.arange(1, 8) + 5, n - 1 - np.arange(300)):
        angle = np.outer(pos.astype(np.float64), f)
        tol = angle * 32 * 2.0 ** -53 + 2 * math.pi * 2.0 ** -25 + 4 * 2.0 ** -24
        at = torch.from_numpy(pos).cuda()
        for t, want in zip(tables, (np.cos(angle), np.sin(angle))):
            assert (np.abs(t[at].cpu().numpy() - want) <= tol).all()
    del tables, t
    torch.cuda.empty_cache()
