"""The cosines and sines of molora_kv_append by themselves: pairs (1, 0) and (0, 1), which the rotation turns into them without another rounding."""
import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("first", [0, 5000, 1_000_000])
def test_cosines_and_sines(first, interleaved):
    """sincospif is off by one step of its result at most, 2^-24 below 1; the sum that brings in the rest of the angle rounds by half a step more, so
    1.5 * 2^-24, and 2^-40 for the rest's own roundings and for the angle (2^-53 of up to 2^18 turns, in both)."""
    n, dim = 3000, 128
    gen = torch.Generator().manual_seed(1)
    table, pages = R.tables([first + n], 128, gen)
    table[0, :first // 128] = 0                                          # (pages that this call does not touch)
    pages = n // 128 + 3
    table[0, first // 128:] = torch.arange(table.shape[1] - first // 128, dtype=torch.int32)
    zeros = torch.zeros(pages, 1, 128, dim, dtype=torch.uint8, device="cuda")
    cache = M.KVCache(zeros, zeros.clone(), torch.ones(pages, 1, device="cuda"), torch.ones(pages, 1, device="cuda"))
    freq = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -torch.arange(0, dim, 2).double() / dim).float()
    q = torch.zeros(n, 2, dim)
    a, b = (q[..., 0::2], q[..., 1::2]) if interleaved else (q[..., :64], q[..., 64:])
    a[:, 0], b[:, 1] = 1.0, 1.0
    kv = torch.zeros(n, 1, dim, device="cuda")
    out = M.molora_kv_append(kv, kv.clone(), cache, table.cuda(), torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([first + n], dtype=torch.int32).cuda(),
                             q=q.cuda(), inv_freq=freq.cuda(), interleaved=interleaved).cpu().double()
    a, b = (out[..., 0::2], out[..., 1::2]) if interleaved else (out[..., :64], out[..., 64:])
    angle = torch.arange(first, first + n).double()[:, None] * freq.double()
    for got, want in ((a[:, 0], angle.cos()), (b[:, 0], angle.sin()), (a[:, 1], -angle.sin()), (b[:, 1], angle.cos())):
        assert float((got - want).abs().max()) <= 1.5 * 2.0 ** -24 + 2.0 ** -40, float((got - want).abs().max() * 2 ** 24)
