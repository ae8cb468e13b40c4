"""molora_kv_attend on values at the ends of what it takes.  Bounds from _kv_reference.attend."""
import math

import pytest
import torch

from test_gpu_kv_attend import check, problem, run

pytestmark = pytest.mark.gpu

# dim, type, heads, kv_heads, new tokens, tokens: a few rows, a few that fill a unit, many
KINDS = [(128, "bf16", 4, 2, (1,), (300,)), (128, "bf16", 4, 2, (9,), (90,)), (128, "bf16", 8, 1, (4,), (700,)), (128, "bf16", 4, 2, (140,), (300,)),
         (64, "bf16", 4, 2, (9,), (90,)), (64, "f32", 4, 2, (3,), (90,)), (128, "f32", 4, 2, (40,), (90,)),
         (128, "bf16", 16, 8, (640,), (700,))]                           # more units of 32 rows than the kernel for few rows is given


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
@pytest.mark.parametrize("new", [3, 150, 2400])
def test_a_row_that_sees_nothing_is_zero_whatever_its_q(dim, dtype, new):
    p = problem(120, (new,), (new - 2,), 4, 2, dim, 64, dtype)
    p["q"][0], p["q"][1, 2, 5] = math.inf, math.nan
    out, lse = run(p)
    assert bool((out[:2] == 0).all()) and bool((lse[:2] == -math.inf).all()) and bool(out[2:].isfinite().all())

SPREADS = [(80, -80), (-80, 80), (90, -100), (-100, 90), (64, -64), (-64, 64)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("first,then", SPREADS)
def test_scales_of_v_far_apart_with_equal_scores(kind, first, then):
    """Every key has the same weight, whatever the scale of its values."""
    dim, dtype, heads, kv_heads, new, _ = KINDS[kind]
    n = new[0]
    p = problem(130 + kind, new, (n + 255,), heads, kv_heads, dim, 16, dtype)
    pool, table = p["pool"], p["table"][0].long()
    pool.k[:] = 0
    half = len(table) // 2
    pool.v_scale[table[:half]], pool.v_scale[table[half:]] = 2.0 ** first, 2.0 ** then
    out, lse = run(p)
    check(p, out, lse)


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("spread", [(-100, 90), (-64, 64)])
def test_scales_of_v_far_apart_with_scores_and_cut_units(kind, spread):
    """A long sequence that many shares divide, its pieces in scales of their own, beside a short one."""
    dim, dtype, heads, kv_heads, new, _ = KINDS[kind]
    n = new[0]
    length = 12000 if n == 140 else n + (1500 if n > 140 else 6000)      # (140 tokens: so long that they go to the kernel for many rows)
    p = problem(140 + kind, (n, 1), (length, 40), heads, kv_heads, dim, 64, dtype)
    pool = p["pool"]
    pool.v_scale[:] = torch.pow(2.0, torch.randint(spread[0], spread[1] + 1, pool.v_scale.shape, generator=p["gen"]).float())
    long_runs = p["table"][0, :min(48, length // 64 // 2 * 2)].long()                                # and runs of pages of one scale, longer than a share
    half = len(long_runs) // 2
    pool.v_scale[long_runs[:half]], pool.v_scale[long_runs[half:]] = 2.0 ** spread[0], 2.0 ** spread[1]
    out, lse = run(p)
    check(p, out, lse)


@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_scales_of_v_beyond_the_range_count_as_its_ends(kind):
    dim, dtype, heads, kv_heads, new, lens = KINDS[kind]
    p = problem(150 + kind, new, lens, heads, kv_heads, dim, 64, dtype)
    pool = p["pool"]
    pool.v_scale[::2], pool.v_scale[1::2] = 2.0 ** -100, 2.0 ** 90
    want = run(p)
    check(p, *want)
    pool.v_scale[::2], pool.v_scale[1::2] = 2.0 ** -126, 2.0 ** 120
    again = run(p)
    assert torch.equal(want[0], again[0]) and torch.equal(want[1], again[1])
