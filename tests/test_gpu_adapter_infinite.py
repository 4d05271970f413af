"""GPU: infinite and NaN operands of the adapters' passes reach what depends
on them, with the definition's values there, and nothing else."""
import numpy as np
import pytest
import torch

from oracle import adapter as AD
from tests import _adapters as T
from tests._adapters import OFFSET, SEED
from tests._gpu import host, log
from tests.test_gpu_adapter import Case

pytestmark = pytest.mark.gpu

# m and rank: tiles of 16 and of 64 rows, the rows in one piece and in several,
# every padded rank
SIZES = [(24, 16), (40, 72), (300, 24), (300, 136), (700, 40), (700, 72), (900, 256), (2000, 8)]


def _inputs(m, rank):
    """Three adapters of ranks `rank`, 0 and 5, rows in turn."""
    d = T.inputs(m + rank, m, 90, 136, rank, 3, False, False)
    d["index"][:] = np.arange(m) % 3
    d["ranks"] = np.array([rank, 0, 5], np.int32)
    return d


@pytest.mark.parametrize("m,rank", SIZES)
def test_gradients_behind_a_rank_are_zero(m, rank):
    """x and dy of rows whose adapters use less than the rank hold infinities
    and NaN: behind that rank the gradients are zero, and those of the other
    adapter keep their bits."""
    log(f"behind the rank {m} {rank}")
    p = 0.3
    d = _inputs(m, rank)
    clean = Case(d)
    _, t = clean.forward(p)
    grads = clean.backward(t, p)
    kept = AD.factors(m, 136, p, SEED, OFFSET) != 0
    for value in (np.inf, -np.inf, np.nan):
        for name in ("x", "dy"):
            e = dict(d, **{name: d[name].copy()})
            for i in (1, 2, m - 1 - m % 3, m - 2 - m % 3):
                assert d["index"][i] in (1, 2)
                e[name][i, np.flatnonzero(kept[i, :90])[3]] = value
            dx, da, db = Case(e).backward(t, p)
            for l, r in enumerate(d["ranks"]):
                assert not da[l, r:].any() and not db[l, :, r:].any(), (value, name, l)
            assert torch.equal(da[0], grads[1][0]) and torch.equal(db[0], grads[2][0])
            own = torch.from_numpy(d["index"] == 2).cuda()
            assert torch.equal(dx[~own], grads[0][~own])
            # what holds them reaches its adapter
            hit = da if name == "x" else db
            assert not torch.isfinite(hit[2, :5] if name == "x" else hit[2, :, :5]).all()
