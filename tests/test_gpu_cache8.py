"""The latent cache in 8 bits on the GPU: tokens quantised as they enter it, and rows read back."""
import math

import pytest
import torch

import cache8_reference as c8
import serving_reference as ref
from test_gpu_decode import BF16, laga  # noqa: F401  (laga: the fixture)

pytestmark = pytest.mark.gpu


def inputs(M, seed=0, beta=True, far=131072):
    g = torch.Generator().manual_seed(seed + M)
    x = torch.randn(M, 576, generator=g) * (0.5 + 2 * torch.rand(M, 1, generator=g)) + torch.randn(M, 1, generator=g)
    gamma, b = (1 + 0.2 * torch.randn(512, generator=g)).to(BF16), (0.1 * torch.randn(512, generator=g)).to(BF16)
    return x.to(BF16), gamma, b if beta else None, torch.randint(0, far, (M,), generator=g, dtype=torch.int32)


def expected(kv, gamma, beta, pos, rope, eps=1e-5):
    """(rows float64 [M, 576], how far fp32 arithmetic may be from them): the references' bounds without their rounding to bf16."""
    y, _, _, b_y = ref.norm(kv[:, :512].double(), gamma.double(), None if beta is None else beta.double(), eps)
    k, b_k = ref.rotate(kv[:, 512:].double(), pos, rope.freqs.cpu(), rope.mscale, rope.interleaved)
    rows, bound = torch.cat([y, k], 1), torch.cat([b_y, b_k], 1)
    return rows, (bound - ref.U * rows.abs()) / (1 + ref.U)


def check_rows(pages, slots, rows, slack):
    """The rows that the pages hold: a power of two as scale, the smallest that will do, and codes within half a step."""
    codes, scales = c8.planes(pages)
    page = codes.shape[1]
    at = slots.long()
    s = scales[at // page, at % page].double()
    amax, room = rows.abs().amax(1), slack.amax(1)
    assert bool(((s >= c8.scale_of((amax - room).clamp(min=0))) & (s <= c8.scale_of(amax + room))).all())
    assert bool((torch.frexp(s)[0] == 0.5).all())
    held = c8.decode_rows(codes[at // page, at % page], s.float())
    step = torch.full((576,), c8.E, dtype=torch.float64)
    step[512:] = c8.E ** 2
    least = c8.LEAST * s[:, None] * torch.ones(576, dtype=torch.float64)
    bound = step * (rows.abs() + slack) + least + 2 * slack + 2.0 ** -23 * rows.abs()
    assert float(((held - rows).abs() - bound).max()) <= 0


@pytest.mark.parametrize("M,page", [(1, 16), (2, 64), (15, 1024), (16, 32), (17, 128), (333, 16), (5000, 64)])
@pytest.mark.parametrize("interleaved,beta", [(True, True), (False, False)])
def test_append_against_float64(laga, M, page, interleaved, beta):  # noqa: F811
    kv, gamma, b, pos = inputs(M, beta=beta)
    rope = laga.rope_plan(64, scaling={"type": "yarn", "factor": 40} if beta else None, interleaved=interleaved)
    n_pages = -(-M // page) + 3
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(M))[:M].to(torch.int32)
    pages = c8.empty_pages(n_pages, page, 0x5a).cuda()
    wide = torch.full((M, 640), float("nan"), dtype=BF16, device="cuda")      # rows a pitch apart
    wide[:, :576] = kv.cuda()
    got = laga.cache_append(wide[:, :576], gamma.cuda(), None if b is None else b.cuda(), pos.cuda(), rope, slots.cuda(), pages)
    assert got is pages
    pages = pages.cpu()
    rows, slack = expected(kv, gamma, b, pos, rope)
    check_rows(pages, slots, rows, slack)
    codes, scales = c8.planes(pages)
    other = torch.ones(n_pages * page, dtype=torch.bool)
    other[slots.long()] = False
    assert bool((codes.reshape(-1, 640)[other] == 0x5a).all()) and bool((scales.reshape(-1, 1).contiguous().view(torch.uint8)[other] == 0x5a).all())


def test_padding_and_slots_outside_write_nothing(laga):  # noqa: F811
    kv, gamma, _, pos = inputs(40)
    pages = c8.empty_pages(4, 16, 0x11).cuda()
    slots = torch.full((40,), -1, dtype=torch.int32)
    slots[1::4], slots[2::4], slots[3::4] = 64, -2147483648, 2147483647
    laga.cache_append(kv.cuda(), gamma.cuda(), None, pos.cuda(), laga.rope_plan(64), slots.cuda(), pages)
    assert bool((pages == 0x11).all())
    slots[7] = 63
    laga.cache_append(kv.cuda(), gamma.cuda(), None, pos.cuda(), laga.rope_plan(64), slots.cuda(), pages)
    assert int((pages != 0x11).any(1).sum()) == 1 and bool((pages[:3] == 0x11).all())


def test_rows_of_zeros_small_and_huge_channels_and_what_is_not_finite(laga):  # noqa: F811
    """No rotation (position 0), gamma 0, so that a row's channels are beta and its key: all zeros; the key alone; a key 2^30 times the
    latent, and 2^-30 times; the largest bf16; an infinity and a NaN."""
    M = 8
    kv = torch.randn(M, 576, generator=torch.Generator().manual_seed(3)).to(BF16)
    pos = torch.zeros(M, dtype=torch.int32)
    rope = laga.rope_plan(64)
    top = float(torch.finfo(BF16).max)
    for k, value in enumerate([0.0, 1.0, 2.0 ** 30, 2.0 ** -30, top, math.inf, math.nan, 2.0 ** -60]):
        kv[k, 512:] = 0
        kv[k, 515] = value
    kv[2, 516] = 2.0 ** 30 * 1.25
    slots = torch.arange(M, dtype=torch.int32)
    for beta in (0.0, 0.75):
        pages = c8.empty_pages(1, 16).cuda()
        b = torch.full((512,), beta, dtype=BF16)
        laga.cache_append(kv.cuda(), torch.zeros(512, dtype=BF16).cuda(), b.cuda(), pos.cuda(), rope, slots.cuda(), pages)
        latent, k_pe = laga.cache_read(pages, slots.cuda())
        want = torch.cat([b.double().expand(M, -1), kv[:, 512:].double()], 1)
        fine = want.isfinite().all(1)
        assert bool(latent[~fine].isnan().all()) and bool(k_pe[~fine].isnan().all()) and int((~fine).sum()) == 2
        codes, scales = c8.planes(pages.cpu())
        want_codes, want_scales = c8.encode(want[fine])
        assert torch.equal(scales[0, :M][fine], want_scales)
        assert torch.equal(codes[0, :M][fine] & 0x7f, want_codes & 0x7f)          # (zeros may be signed)
        held = c8.decode_rows(want_codes, want_scales)
        assert torch.equal(latent[fine].double().cpu(), held[:, :512]) and torch.equal(k_pe[fine].cpu(), held[:, 512:].to(BF16))
    assert float(scales[0, 0]) == 2.0 ** -9 and float(c8.planes(pages.cpu())[1][0, 4]) == 2.0 ** 120


def test_read_is_exact_for_every_code(laga):  # noqa: F811
    """All 256 codes in every channel class, at scales of 2^-32 to 2^120 and NaN, rows in any order, repeated, and none."""
    for page in (16, 64, 1024):
        n = 2 * 1024 // page
        pages = c8.empty_pages(n, page)
        codes, scales = c8.planes(pages)
        g = torch.Generator().manual_seed(page)
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8))
        flat = scales.shape
        scales.copy_(torch.exp2(torch.randint(-32, 100, flat, generator=g).float()))
        scales[0, 3], scales[-1, -1] = math.nan, 2.0 ** 120
        slots = torch.randint(0, n * page, (3001,), generator=g, dtype=torch.int32)
        slots[:4] = torch.tensor([3, n * page - 1, 0, n * page - 1])
        slots[10:20], slots[20], slots[21] = -1, n * page, -2147483648
        latent, k_pe = torch.full((3001, 512), 7.0, dtype=BF16, device="cuda"), torch.full((3001, 64), 7.0, dtype=BF16, device="cuda")
        a, b = laga.cache_read(pages.cuda(), slots.cuda(), latent=latent, k_pe=k_pe)
        assert a.data_ptr() == latent.data_ptr() and b.data_ptr() == k_pe.data_ptr()
        at = slots.long().clamp(0, n * page - 1)
        rows = c8.decode_rows(codes[at // page, at % page], scales[at // page, at % page]).to(torch.float32)
        rows[(slots < 0) | (slots >= n * page)] = 0
        want = rows.to(BF16)
        got = torch.cat([latent, k_pe], 1).cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0), want.nan_to_num(0))


def test_empty_calls(laga):  # noqa: F811
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    pages = c8.empty_pages(2, 16).cuda()
    latent, k_pe = laga.cache_read(pages, none)
    assert latent.shape == (0, 512) and k_pe.shape == (0, 64)
    gamma = torch.ones(512, dtype=BF16, device="cuda")
    assert laga.cache_append(torch.zeros(0, 576, dtype=BF16, device="cuda"), gamma, None, none, laga.rope_plan(64), none, pages) is pages
    assert bool((pages == 0xff).all())


def test_append_and_read_on_a_side_stream_and_in_a_graph(laga):  # noqa: F811
    kv, gamma, b, pos = (t.cuda() for t in inputs(100))
    rope, slots = laga.rope_plan(64), torch.arange(100, dtype=torch.int32, device="cuda")
    want = laga.cache_append(kv, gamma, b, pos, rope, slots, c8.empty_pages(7, 16).cuda())
    latent, k_pe = laga.cache_read(want, slots)
    side = torch.cuda.Stream()
    pages = c8.empty_pages(7, 16).cuda()
    side.wait_stream(torch.cuda.current_stream())
    laga.cache_append(kv, gamma, b, pos, rope, slots, pages, stream=side)
    l2, k2 = laga.cache_read(pages, slots, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(pages, want) and torch.equal(l2, latent) and torch.equal(k2, k_pe)
    pages.fill_(0xff)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        laga.cache_append(kv, gamma, b, pos, rope, slots, pages)
        l3, k3 = laga.cache_read(pages, slots)
    slots.copy_(slots.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(l3, latent) and torch.equal(k3, k_pe) and not torch.equal(pages, want)


def test_rows_past_four_gigabytes(laga):  # noqa: F811
    """Seven million rows of 644 bytes: pages on both sides of 2^31 and 2^32 bytes, written and read."""
    page, n_pages = 64, 110_000
    cache = torch.zeros(n_pages, page * 644, dtype=torch.uint8, device="cuda")
    edges = [0, 2 ** 31 // (page * 644), 2 ** 32 // (page * 644), 2 ** 32 // (page * 644) + 1, n_pages - 1]
    kv, gamma, b, pos = (t.cuda() for t in inputs(len(edges) * 2))
    slots = torch.tensor([p * page + r for p in edges for r in (0, 63)], dtype=torch.int32, device="cuda")
    rope = laga.rope_plan(64)
    laga.cache_append(kv, gamma, b, pos, rope, slots, cache)
    near = laga.cache_append(kv, gamma, b, pos, rope, torch.arange(len(slots), dtype=torch.int32, device="cuda"), c8.empty_pages(1, 16).cuda())
    here, there = laga.cache_read(cache, slots), laga.cache_read(near, torch.arange(len(slots), dtype=torch.int32, device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(here, there)) and bool(here[0].abs().amax(1).min() > 0)
    used = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    used[edges] = True
    assert not bool(cache[~used].any())
    del cache
    torch.cuda.empty_cache()


def test_refusals(laga):  # noqa: F811
    kv, gamma, b, pos = (t.cuda() for t in inputs(4))
    rope, slots = laga.rope_plan(64), torch.arange(4, dtype=torch.int32, device="cuda")
    pages = c8.empty_pages(2, 16).cuda()
    for bad in (pages[:, :-1], pages.view(2, 16, 644), pages.view(torch.int8), c8.empty_pages(2, 16), pages.t()):
        with pytest.raises((ValueError, TypeError, laga.LagaError)):
            laga.cache_append(kv, gamma, b, pos, rope, slots, bad)
        with pytest.raises((ValueError, TypeError, laga.LagaError)):
            laga.cache_read(bad, slots)
    for tokens in (24, 8, 2048):                             # pages that are none
        with pytest.raises(laga.LagaError):
            laga.cache_read(c8.empty_pages(2, tokens).cuda(), slots)
        with pytest.raises(laga.LagaError):
            laga.cache_append(kv, gamma, b, pos, rope, slots, c8.empty_pages(2, tokens).cuda())
    with pytest.raises(ValueError, match="dense"):
        laga.latent_norm_rope(kv, gamma, b, pos, rope, cache=pages, slots=slots)
    with pytest.raises(ValueError):
        laga.cache_append(kv[:, :320], gamma[:256], None, pos, rope, slots, pages)
    with pytest.raises(ValueError):
        laga.cache_append(kv, gamma, b, pos, rope, slots[:3], pages)
    with pytest.raises(ValueError):
        laga.cache_read(pages, slots.long())
    with pytest.raises(ValueError):
        laga.cache_read(pages, slots, latent=torch.empty(4, 511, dtype=BF16, device="cuda"))
    with pytest.raises(laga.LagaError):                      # the slots inside an output
        out = torch.zeros(4, 64, dtype=BF16, device="cuda")
        laga.cache_read(pages, out.view(-1)[:8].view(torch.int32), k_pe=out)
