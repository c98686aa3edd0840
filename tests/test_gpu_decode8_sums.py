"""One-token attention over the cache in 8 bits, where what a test asks for must show a wrong scale, a lost tile or a stale word: scales far apart with scores of order
one, a million tokens of which some pages differ, calls that follow one another in one workspace."""
import math

import pytest
import torch

import cache8_reference as c8
from parity import f64, rel_l2
from test_gpu_decode import BF16, laga  # noqa: F401  (laga: the fixture)
from test_gpu_decode8 import case, check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h", [4, 16, 32, 64, 70])
@pytest.mark.parametrize("less", [0.0, math.log(64.0)])
def test_scales_far_apart_scores_of_order_one(laga, h, less):  # noqa: F811
    """A tile's tokens have scales from 2^-32 to 2^-1, and like weights: scores come from the keys alone (q_nope is zero), the scales of the large tokens from their
    latents.  Half of the weight is tokens' whose values are nothing, so the sum shows in the result too.  less: nats that the large tokens' scores are
    lowered by, so that tokens of order one are as much of the result as they are."""
    def rows_of(b, rows):
        size = torch.tensor([1.0, 2.0 ** -20, 2.0 ** 6, 2.0 ** -31])[torch.arange(len(rows)) % 4].double()
        rows[:, :512] *= size[:, None]
        rows[:, 512:] *= 0.25 * size[:, None].clamp(max=1)
        rows[:, 512] = torch.where(size == 64, -less * 192 ** 0.5 / 4, 0.0)
        return rows

    q, w, pages, table, n = case([700, 3, 129, 64, 31], h, 16, seed=105, fill=0, rows_of=rows_of)
    q[..., :128] = 0
    q[..., 128] = 4.0
    tensors = (q, w, pages, table, n)
    out, lse = run(laga, tensors)
    check(tensors, out, lse)                            # 5e-3 in the mean square
    # a score is off by 2^-8 of its channels' products' sizes at most, which add up to 0.9 in the mean over the tokens (63 * 0.8 * 0.8 * 0.25 * 1.25 / 192^0.5; the
    # query's own channel, 4, is held exactly); the log-sum-exp by a mean of that
    _, want, _, _ = c8.decode(*tensors, 192 ** -0.5)
    assert float((f64(lse) - want).abs().max()) <= 2.0 ** -8


@pytest.mark.parametrize("h", [5, 16, 32, 64])
def test_a_million_tokens_of_different_pages(laga, h):  # noqa: F811
    """Eight pages in any order, one of them once, with 6.5 nats more than the others: some 40 % of the weight in eight tiles of 8192.  The log-sum-exp is that of the pages'
    own, each asked for alone: the weights are the same but for 2^-22 of the exponential and 2^-20 of its argument on either side, sums in fp32 of some 60
    tiles, 32 lanes and 40 pieces a lane (2^-24 each: 8e-6), together 1e-5, and 2^-22 of the number itself."""
    def rows_of(b, rows):
        rows[:, 512] = 0.0
        rows[7168:, 512] = 6.5 * 192 ** 0.5 / 4
        return rows

    q, w, pages, table, n = case([8192, 8192], h, 1024, seed=106, rows_of=rows_of)
    q[..., 128] = 4.0
    tensors = [t.cuda() for t in (q, w, pages)]
    alone = torch.empty(2, 8, h, device="cuda")
    for b in range(2):
        out = laga.paged_decode(tensors[0][b].expand(8, -1, -1).contiguous(), tensors[1], tensors[2], table[b].view(8, 1).contiguous().cuda(),
                                torch.full((8,), 1024, dtype=torch.int32, device="cuda"), lse=alone[b])
        laga.check_status(out[2])
    g = torch.Generator().manual_seed(h)
    which = torch.randint(0, 7, (2, 1024), generator=g)
    which[0, 517], which[1, 1023] = 7, 7
    far, far_lse = torch.empty(2, h, 128, dtype=BF16, device="cuda"), torch.empty(2, h, device="cuda")
    _, _, ws = laga.paged_decode(*tensors, table.gather(1, which).contiguous().cuda(), (n * 128).cuda(), out=far, lse=far_lse)
    laga.check_status(ws)
    for b in range(2):
        times = torch.bincount(which[b], minlength=8).double()
        want_lse = torch.logsumexp(alone[b].double().cpu() + times.log()[:, None], 0)
        assert float(((far_lse[b].double().cpu() - want_lse).abs() - 2.0 ** -22 * want_lse.abs()).max()) <= 2e-5
        weight = (alone[b].double().cpu() + times.log()[:, None] - want_lse).exp()                # [pages, heads]
        parts = torch.stack([c8.decode(q[b:b + 1], w, pages, table[b:b + 1, p:p + 1], torch.tensor([1024], dtype=torch.int32), 192 ** -0.5)[0][0] for p in range(8)])
        assert rel_l2(far[b], (weight[:, :, None] * parts).sum(0)) <= 5e-3


@pytest.mark.parametrize("h", [16, 32, 64])
def test_calls_one_after_another_in_one_workspace(laga, h):  # noqa: F811
    """Without a wait between them, each over what the one before has left: factors, pieces and sums of the call before must not be seen."""
    sets = []
    for seed, lens in ((107, [300, 70, 1] * 20), (108, [1, 500, 64] * 20), (109, [0, 20, 2000] * 2 + [90] * 54)):
        q, w, pages, table, n = case(lens, h, 32, seed=seed)
        sets.append([t.cuda() for t in (q * (seed - 106), w, pages, table, n)])
    want = [laga.paged_decode(*s)[0] for s in sets]
    torch.cuda.synchronize()
    ws = laga.alloc_workspace(laga.paged_decode_workspace_bytes(60, h, cache8=True))
    got = [[torch.empty_like(want[0]) for _ in sets] for _ in range(40)]
    for row in got:
        for s, out in zip(sets, row):
            laga.paged_decode(*s, out=out, workspace=ws)
    torch.cuda.synchronize()
    for row in got:
        assert all(torch.equal(a, b) for a, b in zip(row, want))
