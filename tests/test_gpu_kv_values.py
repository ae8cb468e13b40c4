"""molora_kv_attend on values at the ends of what it takes.  Bounds from _kv_reference.attend."""
import math

import pytest
import torch

from test_gpu_kv_attend import check, problem, run

pytestmark = pytest.mark.gpu

# dim, type, heads, kv_heads, new tokens, tokens: a few rows, a few that fill a unit, many
KINDS = [(128, "bf16", 4, 2, (1,), (300,)), (128, "bf16", 4, 2, (9,), (90,)), (128, "bf16", 8, 1, (4,), (700,)), (128, "bf16", 4, 2, (140,), (300,)),
         (64, "bf16", 4, 2, (9,), (90,)), (64, "f32", 4, 2, (3,), (90,)), (128, "f32", 4, 2, (40,), (90,))]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("one_sign", [False, True])
def test_a_row_of_q_that_is_not_finite_is_nan(kind, value, one_sign):
    """Its scores are infinities of either sign, or all of one sign: the softmax of either is not a number.  No other row knows of it."""
    dim, dtype, heads, kv_heads, new, lens = KINDS[kind]
    p = problem(110 + kind, new, lens, heads, kv_heads, dim, 64, dtype)
    if one_sign:                                                         # every score of the row the same infinity
        p["pool"].k[..., dim - 28] = (p["pool"].k[..., dim - 28] & 0x3F) | 0x08      # positive, not 0, not NaN
    row, head = new[0] // 2, 1
    clean, z = run(p)
    check(p, clean, z)
    p["q"][row, head, dim - 28] = value
    out, lse = run(p)
    keep = torch.ones(new[0], heads, dtype=torch.bool)
    keep[row, head] = False
    assert torch.equal(out.cpu()[keep], clean.cpu()[keep]) and torch.equal(lse.cpu()[keep], z.cpu()[keep])
    assert bool(out[row, head].isnan().all()) and bool(lse[row, head].isnan())


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32")])
@pytest.mark.parametrize("new", [3, 150])
def test_a_row_that_sees_nothing_is_zero_whatever_its_q(dim, dtype, new):
    p = problem(120, (new,), (new - 2,), 4, 2, dim, 64, dtype)
    p["q"][0], p["q"][1, 2, 5] = math.inf, math.nan
    out, lse = run(p)
    assert bool((out[:2] == 0).all()) and bool((lse[:2] == -math.inf).all()) and bool(out[2:].isfinite().all())
