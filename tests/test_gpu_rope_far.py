"""Rotation at the far ends of the 32-bit positions, and with frequencies above one, against angles reduced in exact arithmetic."""
import math
from fractions import Fraction

import pytest
import torch

from parity import f64
from test_gpu_decode import BF16, laga  # noqa: F401  (laga: the fixture)

pytestmark = pytest.mark.gpu
U = 2.0 ** -8
# pi to 60 digits: 2^31 * 50 radians are 2^34 turns, so 30 digits are left of the fraction
TURN = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494")


def reduced(position, freq):
    """position * freq modulo a turn, in radians: exact but for the last rounding to float64."""
    angle = position * Fraction(freq)
    return float(angle - (angle // TURN) * TURN)


def positions(g):
    ends = [0, 1, -1, 2 ** 31 - 1, 2 ** 31 - 2, -2 ** 31, -2 ** 31 + 1, 2 ** 30, -2 ** 30, 5_000_000, 2 ** 24 + 1]
    return ends + [int(v) for v in torch.randint(-2 ** 31, 2 ** 31, (50,), generator=g)]


@pytest.mark.parametrize("largest", [1.0, 50.0])
@pytest.mark.parametrize("interleaved", [True, False])
def test_rotation_at_any_position(laga, interleaved, largest):  # noqa: F811
    """Bound: an angle off by |position * freq| 2^-52 + 3 pi 2^-24 + 2 pi 2^-32 radians, sine and cosine by 2^-21 more, fp32 products by 2^-23 of
    their magnitude, then the rounding to bf16."""
    g = torch.Generator().manual_seed(6)
    pos = positions(g)
    freqs = [largest * 10000.0 ** (-j / 32) for j in range(32)]
    angle = torch.tensor([[reduced(p, f) for f in freqs] for p in pos], dtype=torch.float64)
    off = torch.tensor([[abs(p * f) * 2.0 ** -52 for f in freqs] for p in pos], dtype=torch.float64)
    off = off + 3 * math.pi * 2.0 ** -24 + 2 * math.pi * 2.0 ** -32 + 2.0 ** -21 + 2.0 ** -23
    plan = laga.RopePlan(torch.tensor(freqs, dtype=torch.float64, device="cuda"), 1.0, interleaved)
    x = torch.randn(len(pos), 3, 64, generator=g).to(BF16)
    at = torch.tensor(pos, dtype=torch.int64).to(torch.int32).cuda()
    pairs = torch.arange(32)
    ia, ib = (2 * pairs, 2 * pairs + 1) if interleaved else (pairs, pairs + 32)

    def check(got, given, sign):
        a, b = given[..., ia].double(), given[..., ib].double()
        shape = (len(pos),) + (1,) * (given.dim() - 2) + (32,)
        c, s, o = angle.cos().view(shape), sign * angle.sin().view(shape), off.view(shape)
        for got_c, want in ((f64(got)[..., ia], a * c - b * s), (f64(got)[..., ib], b * c + a * s)):
            slack = (a.abs() + b.abs()) * o
            assert float(((got_c - want).abs() - slack - U * (want.abs() + slack)).max()) <= 0

    check(laga.rope(x.cuda(), at, plan), x, 1)
    check(laga.rope(x.cuda(), at, plan, inverse=True), x, -1)
    kv = torch.randn(len(pos), 576, generator=g).to(BF16)
    gamma = torch.ones(512, dtype=BF16, device="cuda")
    latent, k_pe, mean, rstd = laga.latent_norm_rope(kv.cuda(), gamma, None, at, plan)
    check(k_pe, kv[:, 512:], 1)
    dkv, _, _ = laga.latent_norm_rope_backward(latent, k_pe, kv.cuda(), gamma, mean, rstd, at, plan)
    check(dkv[:, 512:], k_pe.cpu(), -1)
