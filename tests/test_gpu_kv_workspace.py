"""molora_kv_attend with an upper bound on the new tokens that is above what a step has, in every class of rows; bounds from _kv_reference.attend."""
import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M
from test_gpu_kv_attend import check, problem, run

pytestmark = pytest.mark.gpu

# heads, kv_heads, new tokens, upper bound on them
BOUNDS = [(32, 8, (3,), 8), (32, 8, (5,), 8), (32, 8, (6,), 8), (16, 8, (10,), 14), (8, 1, (2,), 4), (8, 1, (3,), 4), (8, 2, (4,), 6), (8, 2, (3, 1), 9), (4, 4, (1,), 31),
          (4, 1, (7, 0, 1), 40), (8, 1, (1,), 2 ** 40)]


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("heads,kv_heads,new,most", BOUNDS)
def test_more_tokens_allowed_than_there_are(heads, kv_heads, new, most, dim, dtype):
    lens = tuple(n + 300 * (i + 1) for i, n in enumerate(new))
    p = problem(90, new, lens, heads, kv_heads, dim, 64, dtype)
    out, lse = run(p, max_tokens=most)                                   # the binding makes the workspace
    check(p, out, lse)


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32")])
def test_one_workspace_for_steps_of_every_size(dim, dtype):
    """Made once for the most tokens that any step has, used by all smaller ones."""
    heads, kv_heads, most = 8, 2, 40
    ws = torch.empty(M.molora_kv_attend_workspace_bytes(M.BF16 if dtype == "bf16" else M.F32, heads, kv_heads, dim, most), dtype=torch.uint8, device="cuda")
    for n in list(range(1, 12)) + [40]:
        p = problem(91, (n,), (n + 200,), heads, kv_heads, dim, 32, dtype)
        for bound in (n, most):
            out, lse = run(p, max_tokens=bound, ws=ws)
            check(p, out, lse)
