"""GPU: low-rank adapters beside a shared projection, forward and backward,
against the float64 oracle, with bounds derived in tests/_adapters.py."""
import numpy as np
import pytest
import torch

from oracle import adapter as AD
from tests import _adapters as T
from tests._adapters import OFFSET, SEED
from tests._gpu import host, log

pytestmark = pytest.mark.gpu

DRAWS = dict(seed=SEED, offset=OFFSET)


def _dev(v, dtype=None, pitch=0):
    """A NumPy array on the device, matrices in rows of `pitch` more elements
    that hold NaN."""
    if v is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(v)).cuda()
    t = t.to(dtype) if dtype else t
    if pitch:
        big = torch.full((t.shape[0], t.shape[1] + pitch), float("nan"), dtype=t.dtype, device="cuda")
        big[:, :t.shape[1]] = t
        t = big[:, :t.shape[1]]
    return t


def _up8(n):
    return -n % 8


class Case:
    def __init__(self, d, pitch=0):
        import paper_2605_31035_amd as M
        self.d = d
        bf = torch.bfloat16
        self.x = _dev(d["x"], bf, 8 * pitch)
        self.a, self.b = _dev(d["a"], bf), _dev(d["b"], bf)
        self.c, self.dx = _dev(d["c"], pitch=pitch), _dev(d["dx"], pitch=pitch)
        self.dy = _dev(d["dy"], bf, _up8(d["dy"].shape[1]) + 8 * pitch)
        self.kw = dict(scaling=_dev(d["scaling"]), ranks=_dev(d["ranks"]))
        self.plan = M.mixfp4_adapter_plan(_dev(d["index"]), len(d["a"]))

    def forward(self, p, out_dtype=torch.float32, **kw):
        import paper_2605_31035_amd as M
        return M.mixfp4_adapter(self.x, self.a, self.b, self.plan, c=self.c, p=p, out_dtype=out_dtype,
                                keep_t=True, **DRAWS, **self.kw, **kw)

    def backward(self, t, p, **kw):
        import paper_2605_31035_amd as M
        return M.mixfp4_adapter_backward(self.dy, self.x, t, self.a, self.b, self.plan, dx=self.dx, p=p,
                                         **DRAWS, **self.kw, **kw)


def _within(name, got, want, bound):
    got = host(got.double())
    err = abs(got - want)
    bad = ~(err <= bound + 1e-300)
    assert not bad.any(), (f"{name}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}, "
                           f"worst {np.nanmax(err / (bound + 1e-300))} of the bound")


# (m, n, k, rank, adapters, mixed ranks, rows of an adapter together)
SHAPES = [(1, 1, 8, 8, 1, False, True), (1, 64, 64, 16, 3, False, True), (2, 130, 4096, 8, 4, True, False),
          (5, 33, 72, 24, 2, True, False), (16, 257, 256, 64, 1, False, True),
          (17, 130, 136, 40, 5, True, False), (48, 520, 1032, 64, 32, True, False),
          (255, 129, 264, 16, 3, False, True), (256, 200, 512, 32, 3, True, False),
          (333, 1000, 384, 8, 3, True, True), (300, 257, 520, 72, 7, False, False),
          (509, 264, 2056, 32, 6, True, True), (700, 135, 1288, 136, 2, False, True),
          (1030, 300, 1032, 256, 2, False, True), (2049, 96, 264, 64, 40, True, False),
          (2048, 1100, 256, 128, 1, False, True), (4500, 72, 136, 16, 200, True, False),
          (513, 1000, 384, 8, 3, True, True), (768, 129, 264, 16, 1, False, True),
          (640, 200, 512, 32, 3, True, False), (1200, 257, 520, 64, 7, True, False)]


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:5])))
def test_forward_and_backward(shape, p):
    log(f"adapter {shape} p={p}")
    pitch = shape[0] % 2                     # odd m: rows apart, so unaligned fp32 rows
    case = Case(T.inputs(sum(shape[:5]), *shape), pitch)
    for dtype in (torch.float32, torch.bfloat16):
        out, t = case.forward(p, dtype)
        want, wt, eo, et = T.forward_bounds(case.d, p, dtype == torch.bfloat16)
        _within(f"out {dtype}", out, want, eo)
        _within("t", t, wt, et)
    want, bounds = T.backward_bounds(case.d, host(t), p)
    got = case.backward(t, p)
    for name, g, w, e in zip(("dx", "da", "db"), got, want, bounds):
        _within(name, g, w, e)
    # the same calls again give the same bits
    out2, t2 = case.forward(p, torch.bfloat16)
    assert torch.equal(out2, out) and torch.equal(t2, t)
    for g, h in zip(got, case.backward(t, p)):
        assert torch.equal(g, h)


@pytest.mark.parametrize("m", [3, 70, 600, 1500])
def test_no_row_has_an_adapter(m):
    d = T.inputs(m, m, 96, 64, 16, 3, False, False)
    d["index"][:] = np.where(np.arange(m) % 2, -1, 3)
    case = Case(d)
    out, t = case.forward(0.2)
    assert torch.equal(out, case.c) and not t.any()
    dx, da, db = case.backward(t, 0.2)
    assert torch.equal(dx, case.dx) and not da.any() and not db.any()


@pytest.mark.parametrize("m", [24, 300, 700])
def test_rank_zero_and_p_one(m):
    d = T.inputs(m, m, 96, 64, 16, 2, False, False)
    d["ranks"] = np.array([0, -5], np.int32)
    case = Case(d)
    out, t = case.forward(0.0)
    assert torch.equal(out, case.c) and not t.any()
    dx, da, db = case.backward(t, 0.0)
    assert torch.equal(dx, case.dx) and not da.any() and not db.any()
    d["ranks"] = None
    case = Case(d)
    out, t = case.forward(1.0)
    assert torch.equal(out, case.c) and not t.any()
    dx, da, db = case.backward(t, 1.0)
    assert torch.equal(dx, case.dx) and not da.any() and not db.any()


@pytest.mark.parametrize("m,rank", [(20, 16), (40, 72), (400, 16), (600, 16), (700, 136), (900, 64)])
def test_unread_places_hold_anything(m, rank):
    """NaN in dropped elements of x, in rows without an adapter, behind an
    adapter's rank, in adapters that no row has: nothing changes."""
    p = 0.4
    d = T.inputs(m + rank, m, 90, 136, rank, 4, False, False)
    d["index"][d["index"] == 2] = 1
    d["ranks"] = np.array([rank, rank // 2 - 3, 5, 11], np.int32)
    clean = Case(d)
    want, t = clean.forward(p)
    grads = clean.backward(t, p)
    f = AD.factors(m, 136, p, SEED, OFFSET)
    e = {q: (None if v is None else v.copy()) for q, v in d.items()}
    nan = np.float32(np.nan)
    e["x"][f == 0] = nan
    none = (d["index"] < 0) | (d["index"] >= 4)
    assert none.any()
    e["x"][none] = np.inf
    e["dy"][none] = nan
    for l, r in enumerate(d["ranks"]):
        e["a"][l, r:] = nan
        e["b"][l, :, r:] = np.inf
    e["a"][2], e["b"][2], e["scaling"][2] = nan, nan, nan
    dirty = Case(e)
    out, t2 = dirty.forward(p)
    assert torch.equal(out, want) and torch.equal(t2, t)
    tn = t.clone()
    tn[torch.from_numpy(none).cuda()] = float("nan")
    for l, r in enumerate(d["ranks"]):
        rows = torch.from_numpy(np.flatnonzero(d["index"] == l)).cuda()
        tn[rows, int(r):] = float("nan")
    for g, h in zip(dirty.backward(tn, p), grads):
        assert torch.equal(g, h)


@pytest.mark.parametrize("m", [24, 300, 700])
def test_infinite_values_stay_where_they_belong(m):
    d = T.inputs(m, m, 96, 64, 16, 2, False, False)
    d["index"][:] = np.arange(m) % 2
    want, _ = Case(d).forward(0.0)
    d["x"][4, 3] = np.inf
    d["c"][7, 9] = np.nan
    out, t = Case(d).forward(0.0)
    finite = torch.isfinite(out)
    assert not finite[4].any() and not finite[7, 9]
    others = torch.ones_like(finite)
    others[4] = False
    others[7, 9] = False
    assert torch.equal(out[others], want[others])
    # t of the row is infinite, not NaN: x times a finite A
    assert torch.isinf(t[4]).all()


def test_without_c_dx_and_scaling_and_in_place():
    import paper_2605_31035_amd as M
    for m in (9, 300, 600):
        d = T.inputs(m, m, 96, 64, 16, 2, False, False)
        d["scaling"][:] = 1.0
        case = Case(d)
        zero = dict(d, c=np.zeros_like(d["c"]), dx=np.zeros_like(d["dx"]))
        want, t = Case(zero).forward(0.1)
        out = M.mixfp4_adapter(case.x, case.a, case.b, case.plan, p=0.1, **DRAWS)
        assert torch.equal(out, want)
        g = Case(zero).backward(t, 0.1)
        h = M.mixfp4_adapter_backward(case.dy, case.x, t, case.a, case.b, case.plan, p=0.1, **DRAWS)
        for u, v in zip(g, h):
            assert torch.equal(u, v)
        # out = c and out = dx themselves, and outputs in wider rows
        want, _ = case.forward(0.1)
        wide = torch.full((m, 100), 5.0, device="cuda")
        case.forward(0.1, out=wide[:, 1:97])
        assert torch.equal(wide[:, 1:97], want) and (wide[:, 97:] == 5).all() and (wide[:, 0] == 5).all()
        case.forward(0.1, out=case.c)
        assert torch.equal(case.c, want)
        want, _, _ = case.backward(t, 0.1)
        wide = torch.full((m, 72), 5.0, device="cuda")
        case.backward(t, 0.1, out=wide[:, 3:67])
        assert torch.equal(wide[:, 3:67], want) and (wide[:, 67:] == 5).all()
        case.backward(t, 0.1, out=case.dx)
        assert torch.equal(case.dx, want)
        buf = torch.zeros((m + 1, 96), device="cuda")
        case.c = buf[:m]
        with pytest.raises(ValueError, match="shares memory"):
            case.forward(0.1, out=buf[1:])


@pytest.mark.parametrize("rank", [16, 72])
def test_empty_batch(rank):
    import paper_2605_31035_amd as M
    case = Case(T.inputs(1, 5, 40, 64, rank, 3, False, False))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    plan = M.mixfp4_adapter_plan(none, 3)
    out, t = M.mixfp4_adapter(case.x[:0], case.a, case.b, plan, keep_t=True)
    assert out.shape == (0, 40) and t.shape == (0, rank)
    dx, da, db = M.mixfp4_adapter_backward(case.dy[:0], case.x[:0], t, case.a, case.b, plan)
    assert dx.shape == (0, 64) and not da.any() and not db.any()


def test_offsets_past_32_bits():
    """Rows of c and out that start past 2^32 elements."""
    d = T.inputs(8, 3, 64, 64, 8, 1, False, True)
    d["index"][:] = 0
    case = Case(d)
    want, _ = case.forward(0.0)
    pitch = (1 << 31) + 8
    buf = torch.empty(2 * pitch + 128, device="cuda")
    c = torch.as_strided(buf, (3, 64), (pitch, 1))
    out = torch.as_strided(buf, (3, 64), (pitch, 1), 64)
    c.copy_(case.c)
    case.c = c
    # rows side by side in one buffer, which the overlap check cannot tell apart
    with pytest.raises(ValueError, match="shares memory"):
        case.forward(0.0, out=out)
    case.forward(0.0, out=c)
    assert torch.equal(c, want)


def test_input_offsets_past_32_bits():
    """Rows of x, dy and the gradients of x that start past 2^31 elements."""
    d = T.inputs(9, 3, 64, 64, 8, 1, False, True)
    d["index"][:] = 0
    case = Case(d)
    want, t = case.forward(0.1)
    grads = case.backward(t, 0.1)
    pitch = (1 << 31) + 8
    for name in ("x", "dy"):
        far = torch.as_strided(torch.empty(2 * pitch + 64, dtype=torch.bfloat16, device="cuda"), (3, 64),
                               (pitch, 1))
        far.copy_(getattr(case, name))
        setattr(case, name, far)
    out, t2 = case.forward(0.1)
    assert torch.equal(out, want) and torch.equal(t2, t)
    far = torch.as_strided(torch.empty(2 * pitch + 64, device="cuda"), (3, 64), (pitch, 1))
    far.copy_(case.dx)
    case.dx = far
    for g, h in zip(case.backward(t, 0.1, out=far), grads):
        assert torch.equal(g, h)


@pytest.mark.parametrize("mixed", [False, True])
def test_results_past_32_bits(mixed):
    """2^31 results and more: the last rows against the oracle, the rows in
    front of them against the same rows in a batch of their own."""
    import paper_2605_31035_amd as M
    m, n, k = 16400, 131080, 32
    small = T.inputs(10, 40, n, k, 8, 2, mixed, False)
    case = Case(small)
    x = torch.randn((m, k), device="cuda").bfloat16()
    x[-40:] = case.x
    index = torch.zeros(m, dtype=torch.int32, device="cuda")
    index[-40:] = _dev(small["index"])
    plan = M.mixfp4_adapter_plan(index, 2)
    out = torch.empty((m, n), device="cuda")
    M.mixfp4_adapter(x, case.a, case.b, plan, out=out, **case.kw)
    small["c"] = np.zeros_like(small["c"])
    want, _, bound, _ = T.forward_bounds(small, 0.0, False)
    _within("out", out[-40:], want, bound)
    first = M.mixfp4_adapter(x[:64].contiguous(), case.a, case.b, M.mixfp4_adapter_plan(index[:64], 2),
                             **case.kw)
    size = first.abs().max()
    assert (out[:64] - first).abs().max() <= 2.0**-15 * size      # other tiles, another order of sums


@pytest.mark.parametrize("m", [20, 300, 700])
def test_infinite_scaling_stays_with_its_adapter(m):
    """An infinite factor reaches its own adapter's rows and gradients, within
    its rank."""
    d = T.inputs(m + 1, m, 90, 136, 16, 3, False, False)
    d["ranks"] = np.array([16, 5, 9], np.int32)
    want, t = Case(d).forward(0.2)
    grads = Case(d).backward(t, 0.2)
    d["scaling"][1] = np.inf
    case = Case(d)
    out, t2 = case.forward(0.2)
    own = torch.from_numpy(d["index"] == 1).cuda()
    assert torch.equal(t2, t) and torch.equal(out[~own], want[~own]) and not torch.isfinite(out[own]).any()
    dx, da, db = case.backward(t, 0.2)
    assert torch.equal(dx[~own], grads[0][~own])
    for l in (0, 2):
        assert torch.equal(da[l], grads[1][l]) and torch.equal(db[l], grads[2][l])
    assert not da[1, 5:].any() and not db[1, :, 5:].any()


def test_passes_on_two_streams_at_once():
    """Each has its own memory."""
    cases = [Case(T.inputs(20 + i, 700, 300, 520, 32, 3, False, False)) for i in range(2)]
    want = []
    for c in cases:
        out, t = c.forward(0.1)
        want.append((out, t, *c.backward(t, 0.1)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(3):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                out, t = c.forward(0.1)
                got[i].append((out, t, *c.backward(t, 0.1)))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(u, v) for u, v in zip(r, want[i]))


def test_other_stream_and_graphs():
    """A call on another stream, and two captured passes that are replayed
    between eager ones on the same inputs."""
    import paper_2605_31035_amd as M
    for m in (12, 400, 800):
        case = Case(T.inputs(m, m, 200, 264, 16, 3, True, False))
        index = _dev(case.d["index"])
        out, t = case.forward(0.2)
        grads = case.backward(t, 0.2)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            o2, t2 = case.forward(0.2)
            g2 = case.backward(t2, 0.2)
        side.synchronize()
        assert torch.equal(out, o2) and all(torch.equal(g, h) for g, h in zip(grads, g2))

        def step():
            case.plan = M.mixfp4_adapter_plan(index, 3)
            o, t = case.forward(0.2)
            return (o, t, *case.backward(t, 0.2))

        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                r = step()
            graphs.append((g, r))
        for i in range(3):
            case.x.normal_()
            index.copy_(index[torch.randperm(m, device="cuda")])
            want = step()
            for g, r in graphs:
                g.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(u, v) for u, v in zip(r, want)), (m, i)


def test_layer_with_adapters():
    """A 4-bit projection with adapters as it is used: quantized product,
    adapters added in place, dropout into the residual; and back: DGRAD's
    product with the adapters' input gradient added."""
    import paper_2605_31035_amd as M
    m, n, k, rank, adapters, p = 96, 160, 256, 16, 3, 0.1
    d = T.inputs(3, m, n, k, rank, adapters, True, True)
    case = Case(d)
    w = torch.from_numpy(T.bf16(np.random.default_rng(1).normal(size=(n, k)) * 0.05)).cuda().bfloat16()
    fwd_w, bwd_w = M.mixfp4_quantize_2d(w)
    c = M.mixfp4_gemm(M.mixfp4_quantize(case.x), fwd_w, workspace="auto")
    d["c"] = host(c)
    out, t = M.mixfp4_adapter(case.x, case.a, case.b, case.plan, c=c, out=c, p=p, keep_t=True, **DRAWS,
                              **case.kw)
    want, _, bound, _ = T.forward_bounds(d, p, False)
    _within("out", out, want, bound)
    residual = torch.randn((m, n), device="cuda").bfloat16()
    y = M.mixfp4_dropout(out, residual=residual, p=p, seed=7, offset=8, out_dtype=torch.bfloat16)
    yw = AD.dropout(host(out), p, 7, 8, residual=host(residual.double()))
    _within("y", y, yw, (2.0**-8 + 2.0**-20) * (abs(yw) + 2.0**-20 * abs(host(out))) + 2.0**-20)
    dy = M.mixfp4_dropout(case.dy, p=p, seed=7, offset=8)          # the gradient that reaches out
    d["dy"] = host(dy.float())
    case.dy = dy
    dx = M.mixfp4_gemm(M.mixfp4_quantize(dy), bwd_w, workspace="auto")
    d["dx"] = host(dx)
    case.dx = dx
    want, bounds = T.backward_bounds(d, host(t), p)
    for name, g, u, e in zip(("dx", "da", "db"), case.backward(t, p, out=dx), want, bounds):
        _within(name, g, u, e)
