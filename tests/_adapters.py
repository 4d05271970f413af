"""Inputs, oracle results and error bounds shared by the adapter tests."""
import numpy as np

from oracle import adapter as AD

SEED, OFFSET = 0xFEDCBA9876543210, 0x0000000700000003


def bf16(v):
    """float64 -> the nearest bf16 values (ties to even), as float32."""
    b = np.asarray(v, np.float32).view(np.uint32)
    return (((b + 0x7FFF + ((b >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


def inputs(seed, m, n, k, rank, adapters, mixed, runs):
    """x, a, b, c, dy, dx, index, scaling, ranks as NumPy arrays (bf16 values
    as float32).  ``runs``: rows of an adapter stand together, else anywhere.
    Some rows have no adapter."""
    rng = np.random.default_rng(seed)
    index = rng.integers(-1, adapters + 1, m).astype(np.int32)
    index[index == adapters] = rng.choice([-2**31, 2**31 - 1, adapters], (index == adapters).sum())
    if adapters == 1 and m > 2:
        index[rng.random(m) < 0.7] = 0
    if runs:
        index = np.sort(index)
    if m == 1:
        index[0] = adapters - 1
    ranks = rng.integers(0, rank + 3, adapters).astype(np.int32) if mixed else None
    if mixed:
        ranks[-1] = rank
    return dict(x=bf16(rng.normal(size=(m, k))), a=bf16(rng.normal(size=(adapters, rank, k)) / k**0.5),
                b=bf16(rng.normal(size=(adapters, n, rank))), c=rng.normal(size=(m, n)).astype(np.float32),
                dy=bf16(rng.normal(size=(m, n))), dx=rng.normal(size=(m, k)).astype(np.float32),
                index=index, scaling=rng.uniform(0.25, 2.0, adapters).astype(np.float32), ranks=ranks)


# Errors of a kernel that is right.  An fp32 sum of q exact products, in any
# order and with each addition off by a whole step, is within
# (q + 8) 2^-23 sum |terms|.  An operand v in two bf16 terms is within 2^-17 of
# itself: with 2^e <= |v| < 2^(e+1) a step of the first term is 2^(e-7), so the
# rest is at most 2^(e-8); that value is a bf16 itself, and below it a step is
# at most 2^(e-9-7), half of which is 2^(e-17) <= 2^-17 |v|.  In three terms (dA, dB) it is within
# 2^-26 of itself, far below e32.  e32 = 2^-23 is a step relative to the value, for the products with
# s and z and the last addition; a bf16 result adds half its step, 2^-8.
E32 = 2.0**-23
SPLIT = 2.0**-17


def _sum(q):
    return (q + 8) * E32


def forward_bounds(d, p, out16):
    """(out, t, bound of out, bound of t)."""
    kw = dict(scaling=d["scaling"], ranks=d["ranks"], p=p, seed=SEED, offset=OFFSET)
    out, t = AD.forward(d["x"], d["a"], d["b"], d["index"], c=d["c"], **kw)
    _, t_abs = AD.forward(abs(d["x"]), abs(d["a"]), abs(d["b"]), d["index"], **kw)
    k, rank = d["x"].shape[1], d["a"].shape[1]
    et = (_sum(k) + 2 * E32) * t_abs
    # through B: the error of t, and the products' own, in terms of |t| + et
    sizes = dict(d, t=None)
    through = _expand(sizes, et + (SPLIT + 2 * E32 + _sum(2 * rank)) * (abs(t) + et))
    eo = through + 2 * E32 * (abs(out) + through)
    if out16:
        eo = eo + 2.0**-8 * (abs(out) + eo)
    return out, t, eo, et


def _expand(d, t):
    """s_l t |B_l|^T by rows."""
    out = np.zeros((t.shape[0], d["b"].shape[1]))
    for l in range(d["a"].shape[0]):
        rows = np.flatnonzero(d["index"] == l)
        _, bl, r = AD._cut(d["a"], d["b"], d["ranks"], l)
        out[rows] = float(d["scaling"][l]) * (t[rows, :r] @ abs(bl).T)
    return out


def backward_bounds(d, t, p):
    """((dx, da, db), (their bounds)) for the kept t (float32)."""
    kw = dict(scaling=d["scaling"], ranks=d["ranks"], p=p, seed=SEED, offset=OFFSET)
    want = AD.backward(d["dy"], d["x"], t, d["a"], d["b"], d["index"], dx=d["dx"], **kw)
    m, k = d["x"].shape
    n, rank = d["b"].shape[1], d["a"].shape[1]
    size = AD.backward(abs(d["dy"]), abs(d["x"]), abs(t), abs(d["a"]), abs(d["b"]), d["index"], **kw)
    u = _sum(n) + 4 * E32                              # of u, relative to sum |dy||B|
    bounds = ((u + SPLIT + _sum(2 * rank)) * size[0] * (1 + 1e-4) + 2 * E32 * abs(want[0]),
              (u + E32 + _sum(3 * m)) * size[1] * (1 + 1e-4) + E32 * abs(want[1]),
              (3 * E32 + _sum(3 * m)) * size[2] * (1 + 1e-4) + E32 * abs(want[2]))
    return want, bounds
