"""Page tables that share an array: rows and columns between each other's."""
import numpy as np
import pytest

from test_pages_gpu import dev, forked

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


W, ROWS = 6, 12
PARENTS, LENGTHS = [0, 2, 1, 2, 0, 1], [96, 17, 40, 96, 1, 80]
# (parents' rows, children's rows) of an array of 12 rows and 20 columns
APART = {"every other row": (np.s_[0:6:2, :W], np.s_[1:9:2, :W]),
         "columns beside": (np.s_[0:3, :W], np.s_[0:4, W:2 * W]),
         "before": (np.s_[6:9, 3:3 + W], np.s_[2:6, 3:3 + W]),
         "other strides, columns beside": (np.s_[0:9:4, :W], np.s_[0:8:2, 14:14 + W]),
         "between, another stride": (np.s_[0:9:4, 4:4 + W], np.s_[1:12:2, :W]),
         "nothing": (np.s_[0:0, :W], np.s_[0:4, :W])}
OVERLAP = {"the same rows": (np.s_[0:3, :W], np.s_[0:4, :W]), "the last row": (np.s_[0:3, :W], np.s_[2:6, :W]), "one column": (np.s_[0:3, :W], np.s_[0:4, W - 1:2 * W - 1]),
           "one row of two strides": (np.s_[0:9:4, :W], np.s_[2:9:2, :W])}


@pytest.mark.parametrize("other_stream", [False, True])
@pytest.mark.parametrize("where", list(APART))
def test_fork_within_an_array(P, torch, where, other_stream):
    rng = np.random.default_rng(3)
    cache = P.PagedKV(100, 16, 1, 64)
    base = rng.integers(0, 100, (ROWS, 20))
    at, to = APART[where]
    table = base[at]
    n = len(base[to])
    refs = np.bincount(table.ravel(), minlength=100)
    want, want_refs = forked(refs, table.tolist() or [[-1] * W], PARENTS[:n] if len(table) else [-1] * n, LENGTHS[:n], 16)
    d, r = dev(torch, base), dev(torch, refs)
    stream = torch.cuda.Stream() if other_stream else None
    torch.cuda.synchronize()
    cache.fork(r, d[at], dev(torch, PARENTS[:n]), dev(torch, LENGTHS[:n]), out=d[to], stream=stream)
    torch.cuda.synchronize()
    base[to] = want
    assert (d.cpu().numpy() == base).all() and (r.cpu().numpy() == want_refs).all()


@pytest.mark.parametrize("where", list(OVERLAP))
def test_fork_onto_its_own_table_is_refused(P, torch, where):
    cache = P.PagedKV(100, 16, 1, 64)
    base = torch.zeros((ROWS, 20), dtype=torch.int32, device="cuda")
    at, to = OVERLAP[where]
    n = base[to].shape[0]
    for stream in (None, torch.cuda.Stream()):
        with pytest.raises(P.QLinearError) as e:
            cache.fork(dev(torch, [0] * 100), base[at], dev(torch, PARENTS[:n]), dev(torch, LENGTHS[:n]), out=base[to], stream=stream)
        assert e.value.status == P.QL_ERR_INVALID_ARG
