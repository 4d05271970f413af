"""CPU pins of the adapter and dropout oracle (draw layout, gradients by
differences) and of the binding's and the C ABI's refusals."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import adapter as AD
from oracle.philox import philox4x32
from tests._adapters import bf16, inputs

P = ctypes.c_void_p
A16, W = P(0x10000), P(0x20000)


def test_draw_layout():
    """Element by element from the generator itself, a partial last group
    and counters past 32 bits included."""
    seed, offset = 0xFEDCBA9876543210, 0x0000000900000004
    for rows, k, first in ((3, 21, 0), (2, 8, (1 << 33) + 5), (1, 1, 7)):
        d = AD.draws(rows, k, seed, offset, row_index=np.arange(first, first + rows, dtype=np.uint64))
        for i in range(rows):
            for j in range(k):
                g = (first + i) * -(-k // 8) + j // 8
                w = philox4x32(np.array([g & 0xFFFFFFFF, g >> 32, 4, 9], np.uint64),
                               np.array([0x76543210, 0xFEDCBA98], np.uint64))
                assert d[i, j] == (int(w[(j % 8) // 2]) >> (16 * (j % 2))) & 0xFFFF


def test_dropout_definition():
    assert AD.threshold(0.0) == 0 and AD.threshold(1.0) == 65536 and AD.threshold(0.1) == 6554
    x = np.ones((300, 500))
    y = AD.dropout(x, 0.25, 3, 4)
    assert set(np.unique(y)) == {0.0, 4.0 / 3.0}
    assert abs((y == 0).mean() - 0.25) < 5 * (0.25 * 0.75 / y.size) ** 0.5   # five sigma
    assert not AD.dropout(x, 1.0).any() and (AD.dropout(x, 0.0) == x).all()
    x[y == 0] = np.nan
    assert (AD.dropout(x, 0.25, 3, 4) == y).all()


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_gradients_by_differences(p):
    """backward() against central differences of sum(dy out) in float64; the
    map is linear in each argument, so only rounding is left."""
    d = inputs(1, 7, 5, 16, 8, 3, True, False)
    kw = dict(scaling=d["scaling"], ranks=d["ranks"], p=p, seed=5, offset=6)
    x, a, b, dy = (d[v].astype(np.float64) for v in ("x", "a", "b", "dy"))
    _, t = AD.forward(x, a, b, d["index"], **kw)
    grads = AD.backward(dy, x, t, a, b, d["index"], **kw)

    def loss(x, a, b):
        return (dy * AD.forward(x, a, b, d["index"], **kw)[0]).sum()

    for which, g in zip((0, 1, 2), grads):
        args = [x, a, b]
        rng = np.random.default_rng(which)
        for _ in range(3):
            step = rng.normal(size=args[which].shape)
            hi, lo = list(args), list(args)
            hi[which], lo[which] = args[which] + step, args[which] - step
            assert abs((loss(*hi) - loss(*lo)) / 2 - (g * step).sum()) < 1e-9 * abs(g * step).sum()


def test_single_row_by_hand():
    """One row, one adapter of rank 2 in arrays of rank 8."""
    x = np.array([[1.0, 2, 0, 0, 0, 0, 0, 3]])
    a = np.zeros((1, 8, 8))
    a[0, 0, 0], a[0, 0, 1], a[0, 1, 7], a[0, 2:] = 1, 1, 2, np.nan
    b = np.full((1, 2, 8), np.nan)
    b[0, :, 0], b[0, :, 1] = [1, 2], [10, 20]
    out, t = AD.forward(x, a, b, [0], c=[[100.0, 200]], scaling=[0.5], ranks=[2])
    assert t[0].tolist() == [3, 6, 0, 0, 0, 0, 0, 0]
    assert out.tolist() == [[100 + 0.5 * (3 + 60), 200 + 0.5 * (6 + 120)]]
    out, t = AD.forward(x, a, b, [1], c=[[100.0, 200]], ranks=[2])
    assert out.tolist() == [[100, 200]] and not t.any()


# --- refusals: nothing below reaches a GPU ----------------------------------
@pytest.fixture(scope="module")
def lib():
    from paper_2605_31035_amd import _lib
    return _lib.lib


def test_dropout_rejects(lib):
    def f(x=A16, xt=0, ldx=64, res=None, rt=0, ldr=64, out=A16, ot=0, ldo=64, rows=4, k=64, p=0.5):
        return lib.mixfp4_dropout(x, xt, ldx, res, rt, ldr, out, ot, ldo, rows, k, p, 0, 0, None)
    assert f(xt=2) == 4 and f(ot=-1) == 4 and f(res=A16, rt=7) == 4
    for p in (-0.1, 1.5, float("nan"), float("inf")):
        assert f(p=p) == 2, p
    assert f(rows=-1) == 2 and f(k=-8) == 2 and f(k=(1 << 32) + 8) == 2
    assert f(ldx=63) == 2 and f(ldo=63) == 2 and f(res=A16, ldr=63) == 2
    assert f(x=P(0)) == 1 and f(out=P(0)) == 1
    assert f(x=P(0x10002)) == 3 and f(out=P(0x10001), ot=1) == 3 and f(res=P(0x10001), rt=1) == 3
    assert f(rows=0) == 0 and f(k=0) == 0 and f(rows=0, x=P(0)) == 0


def test_plan_rejects(lib):
    n = ctypes.c_int64(-1)
    assert lib.mixfp4_adapter_plan_bytes(-1, 4, ctypes.byref(n)) == 2
    assert lib.mixfp4_adapter_plan_bytes(1 << 29, 4, ctypes.byref(n)) == 2
    assert lib.mixfp4_adapter_plan_bytes(8, 0, ctypes.byref(n)) == 2
    assert lib.mixfp4_adapter_plan_bytes(8, 4097, ctypes.byref(n)) == 2
    assert lib.mixfp4_adapter_plan_bytes(8, 4, None) == 1
    assert lib.mixfp4_adapter_plan_bytes(8, 4, ctypes.byref(n)) == 0 and n.value > 0
    f = lib.mixfp4_adapter_plan
    assert f(A16, 8, 4, A16, n.value - 1, None) == 2
    assert f(None, 8, 4, A16, n.value, None) == 1 and f(A16, 8, 4, None, n.value, None) == 1
    assert f(A16, 8, 4, P(0x10008), n.value, None) == 3
    assert f(P(0x10002), 8, 4, A16, n.value, None) == 3


SHAPES = [dict(n=0), dict(k=0), dict(k=60), dict(rank=4), dict(rank=12), dict(rank=264), dict(m=-1),
          dict(adapters=0), dict(adapters=5000), dict(n=(1 << 22) + 1), dict(k=(1 << 22) + 8)]


def test_adapter_rejects(lib):
    def f(x=A16, ldx=64, a=A16, b=A16, plan=A16, c=A16, ldc=48, m=4, n=48, k=64, rank=16, adapters=2,
          p=0.0, t=None, out=A16, ot=0, ldo=48, ws=W, wb=1 << 30):
        return lib.mixfp4_adapter(x, ldx, a, b, None, None, plan, c, ldc, m, n, k, rank, adapters, p,
                                  0, 0, t, out, ot, ldo, ws, wb, None)
    for kw in SHAPES + [dict(p=2.0), dict(ldx=60), dict(ldx=68), dict(ldc=47), dict(ldo=47), dict(wb=0)]:
        assert f(**kw) == 2, kw
    assert f(ldc=1 << 32) == 2 and f(ldo=1 << 32) == 2 and f(ldx=1 << 32) == 2
    assert f(ot=2) == 4
    for name in ("x", "a", "b", "plan", "out", "ws"):
        assert f(**{name: None}) == 1, name
    for name in ("x", "a", "b", "plan"):
        assert f(**{name: P(0x10008)}) == 3, name
    assert f(c=P(0x10002)) == 3 and f(t=P(0x10002)) == 3 and f(ws=P(0x10040)) == 3
    assert f(m=0) == 0


def test_adapter_backward_rejects(lib):
    def f(dy=A16, lddy=48, x=A16, ldx=64, t=A16, a=A16, b=A16, plan=A16, dx_in=None, lddx_in=64, m=4,
          n=48, k=64, rank=16, adapters=2, p=0.0, dx=A16, lddx=64, da=A16, db=A16, ws=W, wb=1 << 30):
        return lib.mixfp4_adapter_backward(dy, lddy, x, ldx, t, a, b, None, None, plan, dx_in, lddx_in,
                                           m, n, k, rank, adapters, p, 0, 0, dx, lddx, da, db, ws, wb,
                                           None)
    for kw in SHAPES + [dict(p=-1.0), dict(ldx=60), dict(lddy=52), dict(lddy=40), dict(lddx=63),
                        dict(dx_in=A16, lddx_in=63), dict(wb=0)]:
        assert f(**kw) == 2, kw
    for name in ("dy", "x", "t", "a", "b", "plan", "dx", "da", "db", "ws"):
        assert f(**{name: None}) == 1, name
    for name in ("dy", "x", "a", "b", "plan", "da", "db"):
        assert f(**{name: P(0x10008)}) == 3, name
    assert f(ws=P(0x10040)) == 3 and f(t=P(0x10002)) == 3


def test_workspace_size(lib):
    f, b = ctypes.c_int64(-1), ctypes.c_int64(-1)
    call = lib.mixfp4_adapter_workspace_size
    assert call(100, 64, 64, 16, 2, None, None) == 1
    assert call(100, 64, 64, 12, 2, ctypes.byref(f), None) == 2
    assert call(100, 64, 64, 16, 2, ctypes.byref(f), ctypes.byref(b)) == 0
    assert f.value > 0 and b.value > f.value
    assert call(0, 64, 64, 16, 2, ctypes.byref(f), ctypes.byref(b)) == 0      # no rows


def _args():
    bf = torch.bfloat16
    import paper_2605_31035_amd as M
    need = ctypes.c_int64(0)
    M.lib.mixfp4_adapter_plan_bytes(6, 2, ctypes.byref(need))
    return dict(x=torch.zeros((6, 32), dtype=bf), a=torch.zeros((2, 8, 32), dtype=bf),
                b=torch.zeros((2, 24, 8), dtype=bf),
                plan=M.AdapterPlan(torch.zeros(need.value, dtype=torch.uint8), 6, 2))


BAD_WEIGHTS = [
    (dict(a=torch.zeros((2, 8, 40), dtype=torch.bfloat16)), "a must have shape"),
    (dict(a=torch.zeros((2, 8, 32))), "bfloat16"),
    (dict(b=torch.zeros((3, 24, 8), dtype=torch.bfloat16)), "b must have shape"),
    (dict(b=torch.zeros((2, 8, 24), dtype=torch.bfloat16).transpose(1, 2)), "contiguous"),
    (dict(scaling=torch.ones(3)), "scaling must have shape"),
    (dict(scaling=torch.ones(2).double()), "float32"),
    (dict(ranks=torch.ones(2).long()), "int32"),
    (dict(x=torch.zeros((6, 64), dtype=torch.bfloat16)[:, ::2]), "unit stride"),
    (dict(x=torch.zeros((6, 36), dtype=torch.bfloat16)[:, :32]), "multiples of 8"),
    (dict(x=torch.zeros((1, 32), dtype=torch.bfloat16).expand(6, 32)), "overlap"),
    (dict(x=torch.zeros((5, 32), dtype=torch.bfloat16)), "plan is for"),
    (dict(x=torch.zeros(32, dtype=torch.bfloat16)), "2-D"),
    (dict(p=1.5), "0 .. 1"),
    (dict(p=float("nan")), "0 .. 1"),
]


def test_binding_adapter_rejects():
    import paper_2605_31035_amd as M
    out = torch.zeros((6, 24))
    cases = BAD_WEIGHTS + [
        (dict(c=torch.zeros((6, 23)), out=out), "c must have shape"),
        (dict(c=torch.zeros((6, 24)).bfloat16(), out=out), "float32"),
        (dict(out=torch.zeros((6, 25))), "out must have shape"),
        (dict(out=out.half()), "out must be"),
        (dict(out=out, out_dtype=torch.bfloat16), "out must be"),
        (dict(out_dtype=torch.float16), "out_dtype"),
        (dict(plan=(1, 2, 3)), "AdapterPlan"),
        (dict(plan=M.AdapterPlan(torch.zeros(8, dtype=torch.uint8), 6, 2)), "element"),
        (dict(), "CUDA tensor"),
        (dict(out=out), "CUDA tensor"),
    ]
    for kw, msg in cases:
        with pytest.raises(ValueError, match=msg):
            M.mixfp4_adapter(**{**_args(), **kw})
    with pytest.raises(ValueError, match="rank must be"):
        M.mixfp4_adapter(**{**_args(), "a": torch.zeros((2, 12, 32), dtype=torch.bfloat16),
                            "b": torch.zeros((2, 24, 12), dtype=torch.bfloat16)})


def test_binding_backward_rejects():
    import paper_2605_31035_amd as M
    dy = torch.zeros((6, 24), dtype=torch.bfloat16)
    t = torch.zeros((6, 8))
    base = dict(dy=dy, t=t)
    cases = BAD_WEIGHTS + [
        (dict(dy=dy.float()), "dy must be"),
        (dict(dy=dy[:, :23]), "dy must have shape"),
        (dict(t=torch.zeros((6, 16))), "t must have shape"),
        (dict(t=t.bfloat16()), "float32"),
        (dict(dx=torch.zeros((6, 31))), "dx must have shape"),
        (dict(out=torch.zeros((6, 32)).bfloat16()), "out must be"),
        (dict(), "CUDA tensor"),
    ]
    for kw, msg in cases:
        with pytest.raises(ValueError, match=msg):
            M.mixfp4_adapter_backward(**{**_args(), **base, **kw})


def test_binding_plan_and_dropout_reject():
    import paper_2605_31035_amd as M
    for index, msg in ((torch.zeros(4).long(), "int32"), (torch.zeros((2, 2), dtype=torch.int32), "1-D"),
                       (torch.zeros(8, dtype=torch.int32)[::2], "contiguous"),
                       (torch.zeros(4, dtype=torch.int32), "CUDA tensor")):
        with pytest.raises(ValueError, match=msg):
            M.mixfp4_adapter_plan(index, 2)
    with pytest.raises(M.MixFP4Error, match="SHAPE"):
        M.mixfp4_adapter_plan(torch.zeros(4, dtype=torch.int32), 0)
    x = torch.zeros((4, 10))
    for kw, msg in ((dict(p=-0.1), "0 .. 1"), (dict(x=x.half()), "x must be"), (dict(x=x[0]), "2-D"),
                    (dict(x=x[:, ::2]), "unit stride"), (dict(residual=x[:3]), "residual must have shape"),
                    (dict(residual=x.double()), "residual must be"), (dict(out=x[:, :9]), "out must have"),
                    (dict(out=x.clone(), out_dtype=torch.bfloat16), "out must be"),
                    (dict(out_dtype=torch.float16), "out_dtype"),
                    (dict(out=x[:1].expand(4, 10)), "overlap"), (dict(), "CUDA tensor")):
        with pytest.raises(ValueError, match=msg):
            M.mixfp4_dropout(**{"x": x, **kw})


def test_seeds_are_integers():
    from paper_2605_31035_amd import _u64
    assert _u64(-1) == 2**64 - 1 and _u64(2**64 + 3) == 3 and _u64(np.int32(5)) == 5
    with pytest.raises(TypeError):
        _u64(1.5)


def test_outputs_apart_from_inputs():
    """An output is an input itself or shares nothing with it."""
    from paper_2605_31035_amd import _apart
    big = torch.zeros((10, 10))
    x, shifted, same = big[:4], big[2:6], big[:4]
    _apart(same, ("x", x), same=x)
    _apart(big[4:8], ("x", x), same=x)
    for out, s in ((shifted, x), (same, None), (big[:4, :9], x), (big.view(-1)[1:41].view(4, 10), x)):
        with pytest.raises(ValueError, match="shares memory"):
            _apart(out, ("x", x), same=s)


def test_bf16_helper():
    v = np.random.default_rng(0).normal(size=1000)
    assert (bf16(v) == torch.from_numpy(v).float().bfloat16().float().numpy()).all()
