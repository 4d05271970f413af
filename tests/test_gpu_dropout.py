"""GPU: dropout without a stored mask against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import adapter as AD
from tests._adapters import E32, OFFSET, SEED
from tests._gpu import host, log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _make(seed, shape, dtype, pitch=0):
    rng = np.random.default_rng(seed)
    big = torch.zeros((shape[0], shape[1] + pitch), dtype=dtype, device="cuda")
    big[:, :shape[1]] = torch.from_numpy(rng.normal(size=shape)).to("cuda").to(dtype)
    return big[:, :shape[1]]


def _f64(t):
    return None if t is None else host(t.double())


def _check(y, x, residual, p, seed=SEED, offset=OFFSET):
    """One multiplication by z (itself rounded) and one addition in fp32, each
    within half a step, 2^-24; a bf16 result rounds once more, 2^-8."""
    want = AD.dropout(_f64(x), p, seed, offset, residual=_f64(residual))
    scaled = abs(AD.dropout(_f64(x), p, seed, offset))
    bound = 2.0**-23 * scaled + 2.0**-24 * abs(want) + 2.0**-40 * (scaled + abs(want))
    if y.dtype == BF16:
        bound = bound + 2.0**-8 * (abs(want) + bound)
    err = abs(_f64(y) - want)
    assert (err <= bound).all(), (err - bound).max()


@pytest.mark.parametrize("xt,rt,ot", [(F32, None, F32), (BF16, None, BF16), (F32, BF16, BF16),
                                      (BF16, F32, F32), (F32, F32, BF16), (BF16, BF16, F32)])
@pytest.mark.parametrize("rows,k,pitch", [(1, 1, 0), (1, 16, 0), (3, 7, 2), (5, 64, 8), (7, 4099, 0),
                                          (33, 129, 3), (300, 256, 4)])
def test_dropout(xt, rt, ot, rows, k, pitch):
    import paper_2605_31035_amd as M
    log(f"dropout {rows}x{k}+{pitch} {xt} {rt} {ot}")
    x = _make(rows + k, (rows, k), xt, pitch)
    r = _make(rows * k, (rows, k), rt, 2 * pitch) if rt else None
    for p in (0.0, 0.1, 0.5, 1.0):
        y = M.mixfp4_dropout(x, residual=r, p=p, seed=SEED, offset=OFFSET, out_dtype=ot)
        assert y.dtype == ot and y.is_contiguous()
        _check(y, x, r, p)


def test_default_type_pitched_out_and_in_place():
    import paper_2605_31035_amd as M
    x = _make(1, (9, 40), BF16)
    assert M.mixfp4_dropout(x, p=0.3).dtype == BF16
    big = torch.full((9, 56), 7.0, device="cuda")
    M.mixfp4_dropout(x, p=0.3, seed=1, offset=2, out=big[:, 8:48])
    _check(big[:, 8:48], x, None, 0.3, 1, 2)
    assert (big[:, :8] == 7).all() and (big[:, 48:] == 7).all()
    for res in (False, True):
        y, r = x.clone(), _make(2, (9, 40), BF16)
        keep = r.clone()
        M.mixfp4_dropout(y, residual=r, p=0.3, seed=1, offset=2, out=r if res else y)
        _check(r if res else y, x, keep, 0.3, 1, 2)
    with pytest.raises(ValueError, match="shares memory"):
        M.mixfp4_dropout(big[:8], out=big[1:])
    e = torch.empty((0, 40), device="cuda")
    assert M.mixfp4_dropout(e, p=0.5).shape == (0, 40)


def test_masked_places_hold_anything():
    """What is dropped may be infinite or NaN; what is kept passes it on."""
    import paper_2605_31035_amd as M
    f = AD.factors(50, 72, 0.4, SEED, OFFSET)
    for dtype in (F32, BF16):
        x = _make(3, (50, 72), dtype)
        want = M.mixfp4_dropout(x, p=0.4, seed=SEED, offset=OFFSET)
        dropped = torch.from_numpy(f == 0).cuda()
        x[dropped] = float("nan")
        assert torch.equal(M.mixfp4_dropout(x, p=0.4, seed=SEED, offset=OFFSET), want)
        i, j = np.argwhere(f != 0)[5]
        x[i, j] = float("-inf")
        y = M.mixfp4_dropout(x, p=0.4, seed=SEED, offset=OFFSET)
        assert y[i, j] == float("-inf") and torch.isfinite(y).sum() == y.numel() - 1
    nan = torch.full((4, 16), float("nan"), device="cuda")
    assert not M.mixfp4_dropout(nan, p=1.0).any()


def test_rows_past_32_bits():
    """Element offsets and group numbers past 2^32: the last rows of a matrix
    of 2^33 + elements, checked by themselves."""
    import paper_2605_31035_amd as M
    rows, k = (1 << 15) + 2, 1 << 18
    x = torch.zeros((rows, k), dtype=BF16, device="cuda")
    x[-2:] = _make(4, (2, k), BF16)
    y = M.mixfp4_dropout(x, p=0.2, seed=SEED, offset=OFFSET)
    f = AD.factors(2, k, 0.2, SEED, OFFSET, row_index=[rows - 2, rows - 1])
    want = host(x[-2:].double()) * f
    assert (abs(host(y[-2:].double()) - want) <= (2.0**-8 + 2.0**-20) * abs(want)).all()
    assert not y[:-2].any()


@pytest.mark.parametrize("xt,rt,ot", [(F32, None, F32), (F32, BF16, BF16), (BF16, F32, F32),
                                      (BF16, BF16, BF16)])
@pytest.mark.parametrize("k", [16384, 16392, 16385])
def test_larger_than_the_infinity_cache(xt, rt, ot, k):
    """More than 256 MB of operands, in rows of whole accesses and not: the
    first and last rows against the oracle."""
    import paper_2605_31035_amd as M
    rows = (300 << 20) // (k * (xt.itemsize + (rt.itemsize if rt else 0) + ot.itemsize)) + 1
    x, r = (None if t is None else torch.randn((rows, k), device="cuda").to(t) for t in (xt, rt))
    y = M.mixfp4_dropout(x, residual=r, p=0.2, seed=SEED, offset=OFFSET, out_dtype=ot)
    for at in (0, rows - 3):
        f = AD.factors(3, k, 0.2, SEED, OFFSET, row_index=np.arange(at, at + 3))
        scaled = _f64(x[at:at + 3]) * f
        want = scaled + (0.0 if r is None else _f64(r[at:at + 3]))
        bound = 2.0**-23 * abs(scaled) + 2.0**-24 * abs(want) + 2.0**-40 * (abs(scaled) + abs(want))
        if ot == BF16:
            bound = bound + 2.0**-8 * (abs(want) + bound)
        assert (abs(_f64(y[at:at + 3]) - want) <= bound).all()


def test_gradient_is_the_same_call():
    import paper_2605_31035_amd as M
    x, dy = _make(5, (64, 136), F32), _make(6, (64, 136), F32)
    kw = dict(p=0.35, seed=3, offset=1 << 40)
    y = M.mixfp4_dropout(x, residual=_make(7, (64, 136), F32), **kw)
    base = M.mixfp4_dropout(torch.zeros_like(x), residual=_make(7, (64, 136), F32), **kw)
    dx = M.mixfp4_dropout(dy, **kw)
    # <dy, dropout(x)> = <dropout(dy), x>; 64 136 products of size about 1, fp32 steps of y
    a, b = ((y - base).double() * dy.double()).sum(), (dx.double() * x.double()).sum()
    size = ((y.abs() + base.abs()).double() * dy.abs().double()).sum()
    assert abs(a - b) <= 4 * E32 * size


def test_other_stream_and_graph():
    import paper_2605_31035_amd as M
    x, r = _make(8, (130, 520), F32), _make(9, (130, 520), BF16)
    want = M.mixfp4_dropout(x, residual=r, p=0.1, seed=1, offset=2, out_dtype=BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = M.mixfp4_dropout(x, residual=r, p=0.1, seed=1, offset=2, out_dtype=BF16)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = M.mixfp4_dropout(x, residual=r, p=0.1, seed=1, offset=2, out_dtype=BF16)
    for i in range(3):
        x.normal_()
        want = M.mixfp4_dropout(x, residual=r, p=0.1, seed=1, offset=2, out_dtype=BF16)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
