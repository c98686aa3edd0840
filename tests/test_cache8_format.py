"""What a token loses in the 8-bit cache's format, as include/laga.h states it, on numbers chosen to lose most (CPU)."""
import torch

import cache8_reference as c8


def worst():
    """Rows whose largest channel is 448 or little less, so that the scale is 1, and channels of every size between codes, at them and half-way."""
    g = torch.Generator().manual_seed(1)
    x = torch.cat([448 * torch.exp2(-20 * torch.rand(200_000, generator=g, dtype=torch.float64)), torch.arange(1, 4096, dtype=torch.float64) * 2.0 ** -11])
    x = torch.cat([x, -x])[: (2 * 204_095) // 575 * 575].view(-1, 575)
    return torch.cat([x, torch.full((len(x), 1), 448.0, dtype=torch.float64)], 1).roll(1, 1)


def test_what_a_channel_loses():
    rows = worst()
    codes, scales = c8.encode(rows)
    assert bool((scales == 1).all())
    lost = (c8.decode_rows(codes, scales) - rows).abs()
    latent, key, x = lost[:, :512], lost[:, 512:], rows.abs()
    # a latent channel to 2^-4 of itself or 2^-10 of the scale, a key channel to 2^-8 of itself or 2^-10 of the scale, whichever is more
    assert float((latent - torch.clamp(x[:, :512] * 2.0 ** -4, min=2.0 ** -10)).max()) <= 0
    assert float((key - torch.clamp(x[:, 512:] * 2.0 ** -8, min=2.0 ** -10)).max()) <= 0
    # ... and no less: a key channel between 2^-6 and 2^-2 of the scale loses more than 2^-8 of itself
    between = (x[:, 512:] > 2.0 ** -6) & (x[:, 512:] < 2.0 ** -2)
    assert bool((key[between] > x[:, 512:][between] * 2.0 ** -8).any()) and bool((latent > x[:, :512] * 2.0 ** -4.2).any())
