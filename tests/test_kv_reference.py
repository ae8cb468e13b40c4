"""The host-side reference of the 8-bit cache against torch's own e4m3 type and against worked values (no GPU)."""
import math

import torch

import _kv_reference as R


def test_codes_are_torchs_e4m3():
    all_codes = torch.arange(256).to(torch.uint8)
    ref = all_codes.view(torch.float8_e4m3fn).double()
    got = R.decode(all_codes)
    assert torch.equal(got.nan_to_num(-1.0), ref.nan_to_num(-1.0)) and torch.equal(got.isnan(), ref.isnan())
    gen = torch.Generator().manual_seed(3)
    x = torch.cat([torch.randn(4000, generator=gen) * 100, torch.randn(4000, generator=gen) * 0.01, ref.float().nan_to_num(0.0),
                   torch.tensor([0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, 447.9])]).clamp(-448, 448)
    assert torch.equal(R.encode(x.double()), x.to(torch.float8_e4m3fn).view(torch.uint8))
    assert R.encode(torch.tensor([1e9, -math.inf, math.inf], dtype=torch.float64)).tolist() == [0x7E, 0xFE, 0x7E]


def test_scales_are_the_smallest_powers_of_two():
    for amax, want in ((448.0, 1.0), (448.1, 2.0), (447.0, 1.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 2.0 ** -64), (1e-30, 2.0 ** -64), (1e30, 2.0 ** 64)):
        assert R.scale_for(amax) == want


def test_rotation_keeps_lengths_and_turns_by_the_position():
    x = torch.randn(5, 2, 64, dtype=torch.float64)
    f = torch.tensor([1.0, 0.5] + [0.0] * 6)                 # rotary 16
    for inter in (False, True):
        y = R.rotate(x, torch.tensor([0, 1, 2, 3, 4]), f, inter)
        assert torch.equal(y[0], x[0]) and torch.equal(y[..., 16:], x[..., 16:])
        assert torch.allclose(y.square().sum(-1), x.square().sum(-1))
        i, j = (0, 1) if inter else (0, 8)
        a, b = x[2, 0, i], x[2, 0, j]
        assert abs(y[2, 0, i] - (a * math.cos(2) - b * math.sin(2))) < 1e-12 and abs(y[2, 0, j] - (b * math.cos(2) + a * math.sin(2))) < 1e-12
