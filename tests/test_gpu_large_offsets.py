"""Offsets past 31 and 32 bits: a cache of 6 GB, rows of the rotary calls whose elements lie past 2^31, pieces of the decode past 4 GB."""
import pytest
import torch

import serving_reference as ref
from parity import f64
from test_gpu_decode import BF16, case, check, laga, run  # noqa: F401  (laga: the fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def test_cache_of_six_gigabytes(laga):  # noqa: F811
    """5.4 million rows of 1152 bytes: pages on both sides of 2^31 and 2^32 bytes, and of 2^31 elements, written by the append and read by the
    decode."""
    page, n_pages = 64, 84_000
    cache = torch.empty(n_pages, page, 576, dtype=BF16, device="cuda")
    edges = [0, 2 ** 31 // (page * 1152), 2 ** 32 // (page * 1152), 2 ** 32 // (page * 1152) + 1, n_pages - 1, 70_001, 17]
    small = case([64 * len(edges), 100], 16, page, seed=41, fill=0.0)
    q, w, pages, table, n = small
    cache[edges] = 3.0
    far = table.clone()
    for k, p in enumerate(edges):
        cache[p] = pages[table[0, k]].cuda()
        far[0, k] = p
    far[1, :2] = torch.tensor([n_pages - 2, 2 ** 31 // (page * 1152) + 1])
    for k in range(2):
        cache[far[1, k]] = pages[table[1, k]].cuda()
    dev = [t.cuda() for t in (q, w)]
    here, _, ws = laga.paged_decode(*dev, cache, far.cuda(), n.cuda())
    laga.check_status(ws)
    assert torch.equal(here, laga.paged_decode(*dev, pages.cuda(), table.cuda(), n.cuda())[0])
    kv = torch.randn(len(edges), 576, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    slots = torch.tensor([p * page + 5 for p in edges], dtype=torch.int32, device="cuda")
    gamma, pos, rope = torch.ones(512, dtype=BF16, device="cuda"), torch.arange(len(edges), dtype=torch.int32, device="cuda"), laga.rope_plan(64)
    before = cache[edges].clone()
    laga.cache_append(kv, gamma, None, pos, rope, slots, cache)
    latent, k_pe, _, _ = laga.latent_norm_rope(kv, gamma, None, pos, rope)
    before[:, 5] = torch.cat([latent, k_pe], 1)
    assert torch.equal(cache[edges], before)


@pytest.mark.parametrize("interleaved", [True, False])
def test_rope_rows_far_apart(laga, interleaved):  # noqa: F811
    """Rows 2^28 elements apart (half a gigabyte): the last of them begins past 2^31 elements, in place and into rows as far apart; and
    a dense tensor of more than 2^32 bytes."""
    M, pitch = 10, 2 ** 28
    whole = torch.empty((M - 1) * pitch + 2 * 192, dtype=BF16, device="cuda")
    x = whole.as_strided((M, 2, 192), (pitch, 192, 1))
    value = torch.randn(M, 2, 192, generator=torch.Generator().manual_seed(2)).to(BF16)
    x.copy_(value.cuda())
    pos = torch.arange(M, dtype=torch.int32, device="cuda")
    rope = laga.rope_plan(64, interleaved=interleaved)
    near = laga.rope(value.cuda(), pos, rope)
    assert torch.equal(laga.rope(x, pos, rope), near)
    laga.rope(x, pos, rope, y=x)
    assert torch.equal(x, near)
    del whole, x
    M, h = 2 ** 32 // (128 * 384) + 100, 128
    x = torch.zeros(M, h, 192, dtype=BF16, device="cuda")
    rows = torch.tensor([0, 2 ** 31 // (h * 384), 2 ** 31 // (h * 192) - 1, 2 ** 32 // (h * 384), M - 1])
    value = torch.randn(len(rows), h, 192, generator=torch.Generator().manual_seed(3)).to(BF16)
    x[rows.cuda()] = value.cuda()
    pos = torch.arange(M, dtype=torch.int32, device="cuda")
    y = laga.rope(x, pos, rope)[rows.cuda()]
    want, bound = ref.rotate(value.double(), rows.to(torch.int32), rope.freqs.cpu(), 1.0, interleaved)
    assert float(((f64(y) - want).abs() - bound).max()) <= 0


def test_latent_rows_past_four_gigabytes(laga):  # noqa: F811
    """3.8 million tokens: kv_a, its gradient and the latents past 2^32 bytes, forward and backward, against the same rows alone."""
    M = 2 ** 32 // 1152 + 77_000
    g = torch.Generator(device="cuda").manual_seed(4)
    kv = torch.randn(M, 576, generator=g, device="cuda", dtype=BF16)
    gamma, rope = torch.rand(512, generator=g, device="cuda").to(BF16), laga.rope_plan(64)
    pos = torch.arange(M, dtype=torch.int32, device="cuda")
    rows = torch.tensor([0, 5, 2 ** 31 // 1152, 2 ** 32 // 1152, 2 ** 32 // 1152 + 1, M - 1], device="cuda")
    latent, k_pe, mean, rstd = laga.latent_norm_rope(kv, gamma, None, pos, rope)
    few = laga.latent_norm_rope(kv[rows], gamma, None, pos[rows], rope)
    for a, b in zip((latent, k_pe, mean, rstd), few):
        assert torch.equal(a[rows], b)
    dkv, dgamma, _ = laga.latent_norm_rope_backward(latent, k_pe, kv, gamma, mean, rstd, pos, rope, with_beta=False)
    alone = laga.latent_norm_rope_backward(latent[rows], k_pe[rows], kv[rows], gamma, mean[rows], rstd[rows], pos[rows], rope, with_beta=False)
    assert torch.equal(dkv[rows], alone[0]) and bool(dgamma.isfinite().all())


def test_pieces_past_four_gigabytes(laga):  # noqa: F811
    """20000 requests of 128 heads: 5.3 GB of pieces (one per request and CTA boundary), 2.7 GB of absorbed queries; a few requests of each
    region against the same requests alone, which split the contexts elsewhere: both within the bounds of the float64 form."""
    B, h = 20_000, 128
    q, w, cache, table, n = case([3, 40, 17, 1], h, 16, seed=42, fill=0.0)
    pick = torch.arange(B) % 4
    big_q = q[pick].cuda()
    out, lse, ws = laga.paged_decode(big_q, w.cuda(), cache.cuda(), table[pick].contiguous().cuda(), n[pick].contiguous().cuda(),
                                     lse=torch.empty(B, h, device="cuda"))
    laga.check_status(ws)
    assert ws.numel() > 2 ** 32
    for b0 in (0, 7_900, 8_192, 15_900, 16_384, B - 4):
        b0 -= b0 % 4
        check((q, w, cache, table, n), out[b0:b0 + 4], lse[b0:b0 + 4])
    for k in range(4):                             # one tile each: the arithmetic does not depend on where in the batch they are
        assert torch.equal(out[k::4], out[k:k + 1].expand(B // 4, -1, -1))
