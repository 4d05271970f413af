"""Low-rank adapters beside a shared projection and dropout without a stored
mask, as cases that can be timed and checked: adapters of many requests from
one token to a large prefill, their forward and backward pass in training, and
dropout on its own and into a residual.

With adapter l = index[i] of row i (none outside [0, L)), rank r_l <= R, A_l
[R, K], B_l [n, R], scaling s_l, keep_ij = (draw of (i, j) >= thr),
thr = round(65536 p) and z = 65536 / (65536 - thr):

    t_i   = z (keep_i x_i) A_l^T          out_i = c_i + s_l t_i B_l^T
    u_i   = s_l dy_i B_l                  dx_i  = dx0_i + z keep_i (u_i A_l)
    dA_l  = z sum u_i^T (keep_i x_i)      dB_l  = s_l sum dy_i^T t_i
    dropout: y = residual + z keep x

The draw of element (i, j) of a [rows, k] matrix is a 16-bit half of
Philox4x32-10 under the key `seed` and the counter (i ceil(k / 8) + j div 8,
offset): with e = j mod 8, the low (e even) or high half of word e div 2.

`listed()` are fixed cases, `draw(rng)` gives more of the same ranges,
`prepare(case, seed)` makes what a program holds before the call, `run(state)`
is one pass, `work(case)` the bytes and operations the pass cannot do without
and `exact(case, seed)` the result in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2, "none": 0}


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------
def listed():
    return [
        # one token of one request beside a square projection: latency alone
        dict(name="token_adapter", kind="forward", m=1, k=4096, n=4096, rank=16, adapters=8,
             kept=True, mixed=False, p=0.0, save=False, out="fp32"),
        # a decode batch whose requests have adapters of several ranks, some none
        dict(name="decode_adapters", kind="forward", m=48, k=4096, n=11008, rank=64, adapters=32,
             kept=True, mixed=True, p=0.0, save=False, out="bf16"),
        # a chunk of a chunked prefill with an odd number of tokens, its rows grouped in the pass
        dict(name="chunk_adapters", kind="forward", m=509, k=11008, n=4096, rank=32, adapters=6,
             kept=False, mixed=True, p=0.0, save=False, out="fp32"),
        # the prefill of a few long requests, grouped in the pass
        dict(name="prefill_adapters", kind="forward", m=2048, k=4096, n=11008, rank=64, adapters=4,
             kept=False, mixed=False, p=0.0, save=False, out="fp32"),
        # adapters of a large rank, as those that stand in for full training
        dict(name="wide_adapters", kind="forward", m=1537, k=4096, n=4096, rank=256, adapters=2,
             kept=True, mixed=False, p=0.0, save=False, out="bf16"),
        # the forward pass of training one adapter, with dropout on its input
        dict(name="train_forward", kind="forward", m=8192, k=4096, n=14336, rank=64, adapters=1,
             kept=True, mixed=False, p=0.05, save=True, out="fp32"),
        # the backward pass of a small batch that trains three small adapters
        dict(name="small_backward", kind="backward", m=333, k=4096, n=4096, rank=8, adapters=3,
             kept=True, mixed=True, p=0.1),
        # the backward pass of a 7B-class layer
        dict(name="train_backward", kind="backward", m=2048, k=4096, n=11008, rank=16, adapters=2,
             kept=True, mixed=False, p=0.05),
        # the backward pass of a large batch through the same layer as train_forward
        dict(name="large_backward", kind="backward", m=8192, k=4096, n=14336, rank=64, adapters=1,
             kept=True, mixed=False, p=0.05),
        # dropout of a few rows of odd length
        dict(name="small_dropout", kind="dropout", rows=7, k=4099, p=0.1, x="fp32", residual="none",
             out="fp32"),
        # a projection's fp32 output through dropout into a bf16 residual
        dict(name="residual_dropout", kind="dropout", rows=2048, k=4096, p=0.1, x="fp32",
             residual="bf16", out="bf16"),
        # a large gradient or activation through dropout
        dict(name="large_dropout", kind="dropout", rows=16384, k=8192, p=0.1, x="bf16",
             residual="none", out="bf16"),
    ]


LARGEST = 8192 * 4096 * 12 + 8192 * 14336 * 2         # bytes of large_backward, about


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("forward", "forward", "backward", "dropout"))
    while True:
        if kind == "dropout":
            case = dict(kind=kind, rows=_log(rng, 1, 16384), k=_log(rng, 16, 28672),
                        p=rng.choice((0.0, 0.05, 0.1, 0.5)), x=rng.choice(("fp32", "bf16")),
                        residual=rng.choice(("none", "fp32", "bf16")), out=rng.choice(("fp32", "bf16")))
        else:
            case = dict(kind=kind, m=_log(rng, 1, 16384), k=16 * _log(rng, 16, 896),
                        n=_log(rng, 64, 28672), rank=8 * _log(rng, 1, 32), adapters=_log(rng, 1, 64),
                        kept=rng.random() < 0.5, mixed=rng.random() < 0.5,
                        p=rng.choice((0.0, 0.0, 0.05, 0.1)))
            if kind == "forward":
                case.update(save=rng.random() < 0.5, out=rng.choice(("fp32", "bf16")))
            # the plain form computes every adapter for every row
            if case["m"] * case["adapters"] * case["rank"] * (case["k"] + case["n"]) > 2e11:
                continue
        if work(case)["bytes"] <= LARGEST:
            return case


def work(case):
    if case["kind"] == "dropout":
        e = case["rows"] * case["k"]
        return {"bytes": e * (SIZE[case["x"]] + SIZE[case["residual"]] + SIZE[case["out"]]),
                "flops": 2 * e}
    m, k, n, r, ad = (case[v] for v in ("m", "k", "n", "rank", "adapters"))
    # the adapters that the requests are expected to name, and the ranks of a mixed set
    used = ad * (1 - (1 - 1 / (ad + case["mixed"])) ** _requests(case))
    weights = int(used * r * (7 / 12 if case["mixed"] else 1)) * (k + n)
    if case["kind"] == "forward":
        b = m * k * 2 + m * n * (4 + SIZE[case["out"]]) + weights * 2 + (m * r * 4 if case["save"] else 0)
        return {"bytes": b, "flops": 2 * m * r * (k + n)}
    b = m * n * 2 + m * k * 10 + m * r * 4 + weights * 2 + ad * r * (k + n) * 4
    return {"bytes": b, "flops": 4 * m * r * (k + n)}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _bf16(g, rows, cols, std, pitch=None):
    """bf16 [rows, cols] in rows of a multiple of 8 elements, a few channels larger than the rest."""
    pitch = pitch or -(-cols // 8) * 8
    t = torch.randn((rows, pitch), generator=g, device=DEV) * std
    t *= torch.exp(0.5 * torch.randn((1, pitch), generator=g, device=DEV))
    return t.to(torch.bfloat16)[:, :cols]


def _requests(case):
    """A decode batch holds one row of each request; in a prefill and in training the rows of a
    request stand together."""
    return case["m"] if case["m"] <= 64 else min(case["m"], 2 * case["adapters"] + 1)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ seed, (seed << 33) | 5
    if case["kind"] == "dropout":
        rows, k = case["rows"], case["k"]
        s["x"] = torch.randn((rows, k), generator=g, device=DEV).to(DTYPES[case["x"]])
        s["residual"] = None
        if case["residual"] != "none":
            s["residual"] = (3 * torch.randn((rows, k), generator=g, device=DEV)).to(
                DTYPES[case["residual"]])
        return s
    m, k, n, r, ad = (case[v] for v in ("m", "k", "n", "rank", "adapters"))
    host = np.random.default_rng(seed)
    requests = _requests(case)
    cuts = np.sort(host.choice(np.arange(1, m), requests - 1, replace=False)) if requests > 1 else []
    which = host.integers(-1 if case["mixed"] else 0, ad, requests)
    s["index"] = torch.from_numpy(np.repeat(which, np.diff([0, *cuts, m])).astype(np.int32)).to(DEV)
    s["ranks"] = None
    if case["mixed"]:                        # smaller adapters stand in the same arrays, the rest zero
        ranks = host.choice([r, max(1, r // 2), max(1, r // 4)], ad)
        s["ranks"] = torch.from_numpy(ranks.astype(np.int32)).to(DEV)
    s["scaling"] = torch.from_numpy((16.0 / r * host.uniform(0.5, 2.0, ad)).astype(np.float32)).to(DEV)
    x = _bf16(g, m, k, 1.0)
    a = (torch.rand((ad, r, k), generator=g, device=DEV) * 2 - 1) * math.sqrt(3.0 / k)
    b = torch.randn((ad, n, r), generator=g, device=DEV) * 0.02
    if s["ranks"] is not None:
        there = torch.arange(r, device=DEV)[None] < s["ranks"][:, None]
        a *= there[:, :, None]
        b *= there[:, None, :]
    s["x"], s["a"], s["b"] = x, a.to(torch.bfloat16), b.to(torch.bfloat16)
    if case["kind"] == "forward":
        s["c"] = torch.randn((m, n), generator=g, device=DEV)      # the shared projection's output
    else:
        s["dy"] = _bf16(g, m, n, 1e-3)
        s["dx"] = torch.randn((m, k), generator=g, device=DEV) * 1e-3   # its gradient's
        s["t"] = _shrink(s)[0]                                     # as the forward pass kept it
    s["plan"] = None
    if case["kept"] and own:                 # a program keeps it over the layers of a batch
        import paper_2605_31035_amd as M
        s["plan"] = M.mixfp4_adapter_plan(s["index"], ad)
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "dropout":
        keep, z = _keep(s["x"].shape, s["p"], s["seed"], s["offset"])
        y = torch.where(keep, s["x"].float() * z, 0.0)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(DTYPES[s["out"]])
    if s["kind"] == "forward":
        t, every = _shrink(s)
        out = (s["c"] + (every * _columns(s["scaling"], s["rank"])) @ _flat_b(s)).to(DTYPES[s["out"]])
        return (out, t) if s["save"] else out
    mine = _mine(s)
    scale = _columns(s["scaling"], s["rank"])
    dy, x, flat_b = s["dy"].float(), s["x"].float(), _flat_b(s)
    keep, z = _keep(x.shape, s["p"], s["seed"], s["offset"])
    u = torch.where(mine, (dy @ flat_b.t()) * scale, 0.0)
    dx = s["dx"] + torch.where(keep, (u @ _flat_a(s)) * z, 0.0)
    da = (u.t() @ torch.where(keep, x, 0.0)) * z
    t = torch.where(mine, s["t"].repeat(1, s["adapters"]), 0.0)
    db = (t * scale).t() @ dy
    return (dx, da.view(s["a"].shape),
            db.view(s["adapters"], s["rank"], s["n"]).transpose(1, 2).contiguous())


def _run_own(s):
    import paper_2605_31035_amd as M
    draws = dict(p=s["p"], seed=s["seed"], offset=s["offset"])
    if s["kind"] == "dropout":
        return M.mixfp4_dropout(s["x"], residual=s["residual"], out_dtype=DTYPES[s["out"]], **draws)
    plan = s["plan"]
    if plan is None:
        plan = M.mixfp4_adapter_plan(s["index"], s["adapters"])
    kw = dict(scaling=s["scaling"], ranks=s["ranks"], **draws)
    if s["kind"] == "forward":
        return M.mixfp4_adapter(s["x"], s["a"], s["b"], plan, c=s["c"], out_dtype=DTYPES[s["out"]],
                                keep_t=s["save"], **kw)
    return M.mixfp4_adapter_backward(s["dy"], s["x"], s["t"], s["a"], s["b"], plan, dx=s["dx"], **kw)


# the plain form: every adapter for every row, and what is not a row's own taken out
def _columns(v, rank):
    return v.repeat_interleave(rank)[None]


def _mine(s):
    return s["index"][:, None] == _columns(torch.arange(s["adapters"], device=DEV), s["rank"])


def _flat_a(s):
    return s["a"].float().reshape(-1, s["k"])


def _flat_b(s):
    return s["b"].float().transpose(1, 2).reshape(-1, s["n"])


def _shrink(s):
    """t [m, rank], and the same in the columns of each row's own adapter among all of them."""
    keep, z = _keep(s["x"].shape, s["p"], s["seed"], s["offset"])
    x = torch.where(keep, s["x"].float(), 0.0)
    every = torch.where(_mine(s), (x @ _flat_a(s).t()) * z, 0.0)
    return every.view(-1, s["adapters"], s["rank"]).sum(1), every


def _keep(shape, p, seed, offset):
    """(which elements dropout keeps, the factor of those)."""
    thr = round(p * 65536)
    z = 65536 / (65536 - thr)
    if thr == 0:
        return torch.ones((1, 1), dtype=torch.bool, device=DEV), z
    rows, k = shape
    groups = -(-k // 8)
    low = 0xFFFFFFFF
    g = torch.arange(rows * groups, device=DEV)
    c0, c1 = g & low, g >> 32
    c2, c3 = torch.full_like(g, offset & low), torch.full_like(g, offset >> 32 & low)
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):                      # the rounds of Philox4x32-10
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (p1 >> 32 & low) ^ c1 ^ k0, p1 & low, (p0 >> 32 & low) ^ c3 ^ k1, p0 & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    words = torch.stack((c0, c1, c2, c3), 1)
    halves = torch.stack((words & 0xFFFF, words >> 16), 2).view(rows, groups * 8)
    return halves[:, :k] >= thr, z


# --------------------------------------------------------------------------
# the definition in 64 bits, adapter by adapter
# --------------------------------------------------------------------------
def _kept64(rows, k, p, seed, offset):
    """fp64 [rows, k]: 1 / (1 - p) (as rounded to 1 / 65536) where kept, 0 elsewhere."""
    thr = int(math.floor(p * 65536 + 0.5))
    if not thr:
        return torch.ones((rows, k), dtype=torch.float64, device=DEV)
    groups = (k + 7) // 8
    u = np.uint64
    mask, sh = u(0xFFFFFFFF), u(32)
    draws = np.empty((rows * groups, 8), np.uint16)
    for first in range(0, rows * groups, 1 << 16):          # pieces that stay in the caches
        g = np.arange(first, min(first + (1 << 16), rows * groups), dtype=u)
        ctr = [g & mask, g >> sh, np.full_like(g, offset & 0xFFFFFFFF),
               np.full_like(g, (offset >> 32) & 0xFFFFFFFF)]
        key = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
        for _ in range(10):
            a, b = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
            ctr = [(b >> sh) ^ ctr[1] ^ u(key[0]), b & mask, (a >> sh) ^ ctr[3] ^ u(key[1]), a & mask]
            key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
        for w in range(4):
            draws[first:first + len(g), 2 * w] = ctr[w] & u(0xFFFF)
            draws[first:first + len(g), 2 * w + 1] = ctr[w] >> u(16)
    kept = torch.from_numpy(draws.reshape(rows, groups * 8)[:, :k] >= thr).to(DEV)
    return kept.double() * (65536.0 / (65536 - thr))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "dropout":
        y = s["x"].double() * _kept64(case["rows"], case["k"], case["p"], s["seed"], s["offset"])
        return y if s["residual"] is None else y + s["residual"].double()
    w = _kept64(case["m"], case["k"], case["p"], s["seed"], s["offset"])
    x = s["x"].double() * w
    forward = case["kind"] == "forward"
    if forward:
        out = s["c"].double()
        t = torch.zeros((case["m"], case["rank"]), dtype=torch.float64, device=DEV)
    else:
        dx = s["dx"].double()
        da = torch.zeros(s["a"].shape, dtype=torch.float64, device=DEV)
        db = torch.zeros(s["b"].shape, dtype=torch.float64, device=DEV)
    for l in range(case["adapters"]):
        rows = torch.nonzero(s["index"] == l)[:, 0]
        if not len(rows):
            continue
        a, b, f = s["a"][l].double(), s["b"][l].double(), float(s["scaling"][l])
        if forward:
            t[rows] = x[rows] @ a.t()
            out[rows] += f * (t[rows] @ b.t())
        else:
            dy = s["dy"][rows].double()
            u = f * (dy @ b)
            dx[rows] += w[rows] * (u @ a)
            da[l] = u.t() @ x[rows]
            db[l] = f * (dy.t() @ s["t"][rows].double())
    if forward:
        return (out, t) if case["save"] else out
    return dx, da, db
