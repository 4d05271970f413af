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


def _same(name, got, want, clean):
    """The definition's infinities and NaN, and every finite value as without
    them (it does not depend on them), bit for bit."""
    got = host(got)
    inf, nan = np.isinf(want), np.isnan(want)
    assert inf.any()
    assert (got[inf] == want[inf]).all(), f"{name}: {(got[inf] != want[inf]).sum()} of {inf.sum()} infinities"
    assert np.isnan(got[nan]).all(), name
    rest = ~(inf | nan)
    assert (got[rest] == host(clean)[rest]).all(), name


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,rank", SIZES)
def test_infinite_operands_forward(m, rank, out_dtype):
    """t enters the wide product in two terms, the second of either sign or
    zero: an infinite element of B times t is infinite all the same, and so is
    one of x behind a rank of one."""
    log(f"infinite forward {m} {rank} {out_dtype}")
    d = _inputs(m, rank)
    d["ranks"][1] = 1
    d["x"][3] = 0.0
    d["x"][3, 0] = 1.0                       # t of row 3 has an element of one term, 1.0
    d["a"][0, 2, 0] = 1.0
    for pitch in (0, 1):
        clean, t = Case(d, pitch).forward(0.0, out_dtype)
        e = dict(d, x=d["x"].copy(), b=d["b"].copy())
        e["x"][4, 11] = np.inf               # adapter 1: t is one infinity
        e["b"][0, 7, 2], e["b"][0, 88, 5], e["b"][1, 8, 0], e["b"][2, 0, 4] = np.inf, -np.inf, np.inf, -np.inf
        e["b"][2, 89, 1], e["b"][2, 89, 3] = np.inf, np.nan
        out, t2 = Case(e, pitch).forward(0.0, out_dtype)
        with np.errstate(invalid="ignore"):
            want, wt = AD.forward(e["x"], e["a"], e["b"], e["index"], c=e["c"], scaling=e["scaling"],
                                  ranks=e["ranks"])
        _same("out", out, want, clean) if out_dtype == torch.float32 else \
            _same("out", out.float(), want, clean.float())
        _same("t", t2, wt, t)
        assert out[3, 7] == np.inf


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("m,rank", SIZES)
def test_infinite_operands_backward(m, rank, p):
    """t and u enter the gradients' products in three terms and dx in two: an
    infinite element of x, dy or A times them is infinite all the same."""
    log(f"infinite backward {m} {rank} p={p}")
    d = _inputs(m, rank)
    d["ranks"][1] = 1
    for pitch in (0, 1):
        case = Case(d, pitch)
        _, t = case.forward(p)
        t[3, 0] = 1.0                        # a row of terms (1, 0, 0)
        clean = case.backward(t, p)
        kept = AD.factors(m, 136, p, SEED, OFFSET) != 0
        for name in ("x", "dy", "a"):
            e = dict(d, **{name: d[name].copy()})
            if name == "a":
                e["a"][0, 3, 5], e["a"][0, 0, 135], e["a"][1, 0, 64], e["a"][2, 4, 0] = np.inf, -np.inf, np.inf, np.nan
            else:
                for i, value in ((3, np.inf), (4, -np.inf), (5, np.inf), (m - 1, -np.inf), (m - 2, np.nan)):
                    e[name][i, np.flatnonzero(kept[i, :90])[i % 7]] = value
            with np.errstate(invalid="ignore"):
                want = AD.backward(e["dy"], e["x"], host(t), e["a"], e["b"], e["index"], dx=e["dx"],
                                   scaling=e["scaling"], ranks=e["ranks"], p=p, seed=SEED, offset=OFFSET)
            got = Case(e, pitch).backward(t, p)
            hits = dict(x=(1,), dy=(0, 1, 2), a=(0,))[name]
            for i, part in enumerate(("dx", "da", "db")):
                if i not in hits:
                    assert torch.equal(got[i], clean[i]), (name, part)
                elif name == "dy" and i < 2:
                    # u of such a row is infinite: what stands beside it is not the clean value's bits,
                    # but the rows and adapters without one are
                    inf, nan = np.isinf(want[i]), np.isnan(want[i])
                    g = host(got[i])
                    assert (g[inf] == want[i][inf]).all() and np.isnan(g[nan]).all(), (name, part)
                    assert np.isfinite(g[~(inf | nan)]).all(), (name, part)
                else:
                    _same(f"{part} of {name}", got[i], want[i], clean[i])


@pytest.mark.parametrize("m,rank", [(24, 16), (24, 72), (600, 24), (600, 200)])
def test_largest_finite_terms(m, rank):
    """t and u between the largest bf16 (255/128 2^127) and the largest fp32:
    their products with small operands are finite, within 2^-17 for the terms
    (2^-16.9 at this end) and a few fp32 steps (2^-21)."""
    import paper_2605_31035_amd as M
    bf = torch.bfloat16
    top, small, tiny = 255 / 128 * 2.0**63, 2.0**56, 2.0**-100
    t_value = 65535 / 32768 * 2.0**127       # (2^64 + 2^56) 255/128 2^63, exact in fp32
    bound = 2.0**-16.9 + 2.0**-21
    plan = M.mixfp4_adapter_plan(torch.zeros(m, dtype=torch.int32, device="cuda"), 1)

    def full(shape, value):
        return torch.full(shape, value, dtype=bf, device="cuda")

    sign = torch.ones((m, 1), device="cuda", dtype=bf)
    sign[::2] = -1
    # t = +-t_value in its first element, zero behind it
    x = torch.zeros((m, 64), dtype=bf, device="cuda")
    x[:, :2] = sign * top
    a = torch.zeros((1, rank, 64), dtype=bf, device="cuda")
    a[0, 0, 0], a[0, 0, 1] = 2.0**64, small
    out, t = M.mixfp4_adapter(x, a, full((1, 40, rank), tiny), plan, keep_t=True)
    s = host(sign.double())
    assert (host(t[:, 0].double()) == s[:, 0] * t_value).all() and not t[:, 1:].any()
    want = s * t_value * tiny
    assert (abs(host(out.double()) - want) <= bound * abs(want)).all()
    # dB from such a t: the sum over the rows, all of one sign
    _, _, db = M.mixfp4_adapter_backward(sign.expand(m, 40).contiguous() * tiny, x, t, a,
                                         full((1, 40, rank), tiny), plan)
    want = m * t_value * tiny
    sums = (m + 8) * 2.0**-23
    assert (abs(host(db[0, :, 0].double()) - want) <= (bound + 3 * sums) * want).all()
    assert not db[0, :, 1:].any()
    # u = +-t_value: dx and dA
    dy = torch.zeros((m, 40), dtype=bf, device="cuda")
    dy[:, :2] = sign * top
    b = torch.zeros((1, 40, rank), dtype=bf, device="cuda")
    b[0, 0, 0], b[0, 1, 0] = 2.0**64, small
    dx, da, _ = M.mixfp4_adapter_backward(dy, sign.expand(m, 64).contiguous() * tiny, torch.zeros_like(t),
                                          full((1, rank, 64), tiny), b, plan)
    assert (abs(host(dx.double()) - s * t_value * tiny) <= bound * t_value * tiny).all()
    assert (abs(host(da[0, 0].double()) - want) <= (bound + 3 * sums) * want).all()
    assert not da[0, 1:].any()
