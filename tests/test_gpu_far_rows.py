"""GPU: batches at the far end of the documented sizes."""
import numpy as np
import pytest
import torch

from oracle import adapter as AD
from tests._adapters import OFFSET, SEED
from tests._gpu import host

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    """These batches take up to 125 GB: none of it stays with torch's allocator,
    whose large free blocks other tests would allocate in."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def test_dropout_groups_past_32_bits():
    """2^32 rows and more of one element, each a group of draws: the counter's
    high word counts."""
    import paper_2605_31035_amd as M
    rows = (1 << 32) + 70
    x = torch.zeros((rows, 1), dtype=torch.bfloat16, device="cuda")
    x[:100] = 1.0
    x[-100:] = 1.0
    y = M.mixfp4_dropout(x, p=0.5, seed=SEED, offset=OFFSET, out=x)
    for at in (0, rows - 100):
        f = AD.factors(100, 1, 0.5, SEED, OFFSET, row_index=np.arange(at, at + 100))
        assert (host(y[at:at + 100].double()) == f).all()       # 0 or 2, exact in bf16


def test_adapter_on_the_most_rows():
    """2^28 rows, whose positions in tiles are more than 2^28: every row of t and
    out, exact (sums of small whole numbers)."""
    import paper_2605_31035_amd as M
    rows, bf = 1 << 28, torch.bfloat16
    value = torch.arange(rows, dtype=torch.int32, device="cuda") % 251
    index = value % 3 - 1                    # none, 0 and 1
    x = value.to(bf)[:, None].expand(rows, 8).contiguous()      # 0 .. 250 are exact
    a = torch.zeros((2, 8, 8), dtype=bf, device="cuda")
    a[0, 0, 3], a[1, 0, 7], a[1, 1, 2] = 1.0, 2.0, -1.0
    b = torch.zeros((2, 1, 8), dtype=bf, device="cuda")
    b[0, 0, 0], b[1, 0, 0], b[1, 0, 1] = 4.0, 1.0, 8.0
    plan = M.mixfp4_adapter_plan(index, 2)
    out, t = M.mixfp4_adapter(x, a, b, plan, keep_t=True)
    del x, plan
    zero = torch.zeros_like(value)
    first = torch.where(index == 0, value, torch.where(index == 1, 2 * value, zero))
    second = torch.where(index == 1, -value, zero)
    assert torch.equal(t[:, 0], first.float()) and torch.equal(t[:, 1], second.float())
    assert not t[:, 2:].any()
    want = torch.where(index == 0, 4 * value, torch.where(index == 1, -6 * value, zero))
    assert torch.equal(out[:, 0], want.float())


def test_adapter_backward_on_the_most_rows():
    """The same for the backward pass: dx of every row, and gradients whose sums
    a few rows at both ends make up."""
    import paper_2605_31035_amd as M
    rows, bf = 1 << 28, torch.bfloat16
    value = torch.arange(rows, dtype=torch.int32, device="cuda") % 5
    index = value - 3                        # none for 0 .. 2, then 0 and 1
    dy = value.to(bf)[:, None].expand(rows, 8).contiguous()[:, :1]
    some = torch.tensor([3, 4, 8, rows - 30, rows - 27, rows - 3, rows - 2, rows - 1], device="cuda")
    x = torch.zeros((rows, 8), dtype=bf, device="cuda")
    t = torch.zeros((rows, 8), device="cuda")
    x[some, 5], t[some, 1] = 2.0, 3.0
    a = torch.zeros((2, 8, 8), dtype=bf, device="cuda")
    a[0, 0, 3], a[1, 1, 7] = 1.0, 2.0
    b = torch.zeros((2, 1, 8), dtype=bf, device="cuda")
    b[0, 0, 0], b[1, 0, 1] = 4.0, -1.0
    plan = M.mixfp4_adapter_plan(index, 2)
    dx, da, db = M.mixfp4_adapter_backward(dy, x, t, a, b, plan)
    del plan, dy, x, t
    zero = torch.zeros_like(value)
    for column, want in ((3, torch.where(index == 0, 4 * value, zero)),
                         (7, torch.where(index == 1, -2 * value, zero))):
        assert torch.equal(dx[:, column], want.float())
        dx[:, column] = 0
    assert not dx.any()
    wa, wb = torch.zeros_like(da), torch.zeros_like(db)
    for i in some.tolist():
        v = i % 5
        if v >= 3:
            wa[v - 3, v - 3, 5] += 2 * v * (4 if v == 3 else -1)
            wb[v - 3, 0, 1] += 3 * v
    assert wa.any() and torch.equal(da, wa) and torch.equal(db, wb)
