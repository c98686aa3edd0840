"""One-token attention over the paged latent cache in 8 bits against the explicit form in float64 over what the cache holds."""
import math

import pytest
import torch

import cache8_reference as c8
from parity import f64, rel_l2
from test_gpu_decode import BF16, laga  # noqa: F401  (laga: the fixture)

pytestmark = pytest.mark.gpu


def case(lens, h, page, seed=0, spare=2, fill=0xff, rows_of=None):
    """Pages in random order; everything no token owns holds `fill` (0xff: NaN codes and scales), unused columns of the table nonsense."""
    g = torch.Generator().manual_seed(seed + sum(lens) + h)
    held = [-(-t // page) for t in lens]
    pages = c8.empty_pages(sum(held) + spare, page, fill)
    codes, scales = c8.planes(pages)
    order = torch.randperm(len(pages), generator=g).to(torch.int32).tolist()
    table = torch.full((len(lens), max(1, max(held))), 0x7fffffff, dtype=torch.int32)
    for b, t in enumerate(lens):
        mine = [order.pop() for _ in range(held[b])]
        if not mine:
            continue
        table[b, : held[b]] = torch.tensor(mine, dtype=torch.int32)
        rows = torch.randn(t, 576, generator=g).double() * (0.25 + 2 * torch.rand(t, 1, generator=g).double())
        c, s = c8.encode(rows if rows_of is None else rows_of(b, rows))
        for k, p in enumerate(mine):
            n = min(page, t - k * page)
            codes[p, :n], scales[p, :n] = c[k * page: k * page + n], s[k * page: k * page + n]
    q = torch.randn(len(lens), h, 192, generator=g).to(BF16)
    w = (torch.randn(512, h * 256, generator=g) * 512 ** -0.5).to(BF16)
    return q, w, pages, table, torch.tensor(lens, dtype=torch.int32)


def run(laga, tensors, scale=None):  # noqa: F811
    dev = [t.cuda() for t in tensors]
    B, h = tensors[0].shape[:2]
    out = torch.full((B, h, 128), float("nan"), dtype=BF16, device="cuda")
    lse = torch.full((B, h), float("nan"), device="cuda")
    _, _, ws = laga.paged_decode(*dev, softmax_scale=scale, out=out, lse=lse)
    laga.check_status(ws, where="laga_paged_decode8")
    return out, lse


def check(tensors, out, lse, scale=192 ** -0.5, l2=5e-3):
    want, want_lse, b_out, b_lse = c8.decode(*tensors, scale)
    assert not torch.isnan(f64(out)).any()
    err = (f64(out) - want).abs()
    assert float((err - b_out).max()) <= 0, (float(err.max()), float(b_out.max()))
    # four roundings of at most 2^-8 (queries, probabilities, latent output, result), each at most that / sqrt(3) in the mean square: 4.5e-3
    if float(want.norm()) > 0:
        assert rel_l2(out, want) <= l2
    live = tensors[4] > 0
    assert bool((lse[~live].cpu() == -math.inf).all()) and bool((out[~live] == 0).all())
    assert float(((f64(lse) - want_lse)[live].abs() - b_lse[live]).max()) <= 0 if bool(live.any()) else True


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("h", [1, 16, 24, 40])
def test_lengths_around_every_boundary(laga, h, page):  # noqa: F811
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 191, 192, 193, 200, 255, 256, 257]
    tensors = case(lens, h, page)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("B,h", [(1, 16), (1, 128), (3, 5), (5, 24), (2, 33), (2, 64), (2, 65), (1, 200), (150, 16), (300, 2), (16, 9), (17, 9), (130, 32)])
def test_batches_and_heads(laga, B, h):  # noqa: F811
    g = torch.Generator().manual_seed(B * 7 + h)
    lens = torch.randint(0, 700 if B < 10 else 90, (B,), generator=g).tolist()
    tensors = case(lens, h, 64, seed=1)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("B,h", [(17, 128), (45, 64), (129, 33), (300, 16)])
def test_several_request_tiles_per_head(laga, B, h):  # noqa: F811
    g = torch.Generator().manual_seed(B + h)
    lens = torch.randint(0, 70, (B,), generator=g).tolist()
    lens[-1] = 1500                                     # one request in many pieces, in the last tile
    tensors = case(lens, h, 32, seed=10)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("B,h", [(65, 128), (129, 64), (193, 40), (257, 33), (600, 16), (66, 150), (1300, 7)])
def test_requests_joined_and_projected_apart(laga, B, h):  # noqa: F811
    g = torch.Generator().manual_seed(B + h)
    lens = torch.randint(0, 70, (B,), generator=g).tolist()
    lens[B // 2], lens[-1] = 9000 if h < 64 else 2500, 0     # many pieces; and none
    tensors = case(lens, h, 32, seed=14)
    check(tensors, *run(laga, tensors))


def test_the_same_requests_with_few_others_and_with_many(laga):  # noqa: F811
    """Values that are not finite stay with their request, whichever kernel joins the pieces."""
    h = 64
    q, w, pages, table, lens = case([90, 0, 700, 33] + [5] * 130, h, 16, seed=15)
    codes, scales = c8.planes(pages)
    codes[int(table[2, 0]), 3, 7] = 0x7f
    q[3, 1, 5] = float("nan")
    many, many_lse = run(laga, (q, w, pages, table, lens))
    few, few_lse = run(laga, (q[:40], w, pages, table[:40], lens[:40]))
    assert bool(torch.isnan(many[2].float()).all()) and bool(torch.isnan(many_lse[2]).all()) and bool((many[1] == 0).all())
    assert bool(torch.isnan(many[3, 1].float()).all()) and not bool(torch.isnan(many[3, 2:].float()).any() | torch.isnan(many[4:].float()).any())
    assert torch.equal(torch.isnan(many[:40].float()), torch.isnan(few.float())) and torch.equal(torch.isnan(many_lse[:40]), torch.isnan(few_lse))


@pytest.mark.parametrize("lens,h,page", [([511], 16, 32), ([9001], 16, 64), ([20011, 3], 4, 16), ([12345, 1, 0, 6000], 32, 64), ([12345, 1, 0, 6000], 64, 64),
                                         ([15000, 777], 128, 256)])
def test_long_contexts(laga, lens, h, page):  # noqa: F811
    tensors = case(lens, h, page, seed=2)
    check(tensors, *run(laga, tensors))


def test_all_empty_and_one_token(laga):  # noqa: F811
    tensors = case([0, 0, 0], 16, 64)
    check(tensors, *run(laga, tensors))
    tensors = case([1], 16, 16)
    out, lse = run(laga, tensors)
    check(tensors, out, lse)
    codes, scales = c8.planes(tensors[2])
    p = int(tensors[3][0, 0])
    v = c8.decode_rows(codes[p, :1], scales[p, :1])[:, :512] @ tensors[1].double().view(512, 16, 256)[..., 128:].reshape(512, -1)
    assert rel_l2(out.reshape(1, -1), v) <= 2.0 ** -7       # softmax of one score is 1: the value itself, rounded once, and its joined parts


@pytest.mark.parametrize("h", [16, 32, 64])
@pytest.mark.parametrize("shape", ["up", "down", "alternate", "cliff"])
def test_scores_that_move_the_reference(laga, h, shape):  # noqa: F811
    """Scores that grow along the context by far more than the window of 2^11, fall, alternate in sign, or drop at once for good: the
    rescaling of the accumulator, both ways."""
    ramp = {"up": torch.linspace(0.1, 30, 1536), "down": torch.linspace(30, 0.1, 1536), "alternate": torch.tensor([30.0, -30.0]).repeat(768),
            "cliff": torch.cat([torch.full((100,), 12.0), torch.full((1436,), 1.0)])}[shape].double()
    signs = torch.where(torch.arange(64) % 3 == 0, -1.0, 1.0).double()

    def rows_of(b, rows):
        rows[:, 512:] = signs * ramp[: len(rows), None]
        return rows

    q, w, pages, table, lens = case([1500, 900], h, 64, seed=3, fill=0, rows_of=rows_of)
    q[..., 128:] = (q[..., 128:].float().abs() * signs.float()).to(BF16)
    tensors = (q, w, pages, table, lens)
    check(tensors, *run(laga, tensors))


def test_a_tile_of_one_large_and_many_small_weights(laga):  # noqa: F811
    """One score 13 above all others, its value next to nothing: what comes out is what 2099 weights of 2^-18.76 of it leave.  Its key makes its
    scale 2^7 of theirs, so that in its tile, where its weight times scale is at 2^4 (up to 32 heads) or 2^7, theirs are 2^-21.8 and 2^-18.8: both under
    what the parts hold (2^-15 and 2^-17), and dropped, as documented.  In all other tiles the reference comes down to them.  The 127 of that tile
    are 127 / 2099 = 6.05e-2 of what comes out, with the other roundings' 5e-3 beside them."""
    for h, l2 in ((16, 6.6e-2), (64, 6.6e-2)):
        def rows_of(b, rows):
            rows[:, 512:] = 0.0
            rows[500, 512] = 13.0 * 192 ** 0.5
            rows[:, :512] = rows[:, :512] * 0.25 + 1.0
            rows[500, :512] = 1e-3
            return rows

        q, w, pages, table, lens = case([2100], h, 64, seed=4, fill=0, rows_of=rows_of)
        q[:] = 0
        q[..., 128] = 1.0
        w = w.abs()                                         # (the small weights' values add up)
        tensors = (q, w, pages, table, lens)
        check(tensors, *run(laga, tensors), l2=l2)


def test_scales_far_apart(laga):  # noqa: F811
    """Tokens whose scales differ by 2^40, small beside large: the weights take the scales' part."""
    def rows_of(b, rows):
        size = torch.tensor([1.0, 2.0 ** -20, 2.0 ** 6, 2.0 ** -31])[torch.arange(len(rows)) % 4].double()
        rows[:, :512] *= size[:, None]
        rows[:, 512:] *= size[:, None].clamp(max=1)
        return rows

    # (Latents of 2^6 make scores of 300, which the queries' 2^-8 moves by 1.2 at worst: e^1.2 between two weights.  The bound of each element has
    # that in it, the mean square's 5e-3 is of scores of order one and says nothing here.)
    for h in (16, 64):
        tensors = case([700, 3], h, 16, seed=5, fill=0, rows_of=rows_of)
        check(tensors, *run(laga, tensors), l2=math.inf)


def test_rows_of_zeros(laga):  # noqa: F811
    """A page as LatentCache makes it (zeros, scales too) stands for rows of zeros: uniform weights over nothing."""
    q, w, pages, table, lens = case([200, 40], 16, 64, seed=6, fill=0)
    pages[table[0, 1].long()] = 0
    tensors = (q, w, pages, table, lens)
    check(tensors, *run(laga, tensors))
    pages[:] = 0
    out, lse = run(laga, (q, w, pages, table, lens))
    assert bool((out == 0).all()) and float((lse.cpu().double() - lens.double().log()[:, None]).abs().max()) <= 1e-5


@pytest.mark.parametrize("value", [-1e30, 3e37])
@pytest.mark.parametrize("lens,h,of", [([100, 70], 16, 0), ([20000, 300], 4, 0), ([300, 9000], 40, 0)])
def test_requests_whose_every_score_is_the_same_huge_value(laga, lens, h, of, value):  # noqa: F811
    """Equal weights whatever the scores' size: the mean of the values (which beside such a key are held as zeros)."""
    def rows_of(b, rows):
        if b == of:
            rows[:, 512:] = 0
            rows[:, 515] = value
        return rows

    q, w, pages, table, n = case(lens, h, 16, seed=7, fill=0, rows_of=rows_of)
    q[of] = 0
    q[of, :, 131] = 0.5
    out, lse = run(laga, (q, w, pages, table, n))
    held = c8.decode_rows(*(x[table[of, 0].long()][0] for x in c8.planes(pages)))[515]
    assert bool((out[of] == 0).all())
    score = 0.5 * float(held) * 192 ** -0.5
    assert float(((lse[of].double().cpu() - score) / score).abs().max()) <= 2.0 ** -20      # (log t is nothing beside it)
    live = [b for b in range(len(lens)) if b != of]
    check((q[live], w, pages, table[live], n[live]), out[live], lse[live])


def test_values_that_are_not_finite(laga):  # noqa: F811
    """A NaN among a request's own codes, or scales, or queries, reaches its result; nothing reaches another request's."""
    for h in (16, 64):
        q, w, pages, table, lens = case([100, 130, 64, 300], h, 16, seed=8)
        clean, _ = run(laga, (q, w, pages, table, lens))
        codes, scales = c8.planes(pages)
        codes[int(table[0, 0]), 3, 7] = 0x7f
        scales[int(table[1, 3]), 5] = float("nan")
        q[3, 0, 5] = float("nan")
        q[3, 1, 130] = float("inf")
        out, lse = run(laga, (q, w, pages, table, lens))
        assert bool(torch.isnan(out[:2].float()).all()) and bool(torch.isnan(lse[:2]).all())
        assert bool(torch.isnan(out[3, :2].float()).all()) and torch.equal(out[3, 2:], clean[3, 2:]) and torch.equal(out[2], clean[2])


def test_shared_pages_and_repeated_requests(laga):  # noqa: F811
    q, w, pages, table, _ = case([400], 16, 32, seed=9)
    q = torch.cat([q, torch.randn_like(q.float()).to(BF16), q, q])
    tensors = (q, w, pages, table.expand(4, -1).contiguous(), torch.tensor([400, 333, 400, 400], dtype=torch.int32))
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("h", [16, 64])
def test_bad_pages_and_lengths_are_reported(laga, h):  # noqa: F811
    """A page number outside the cache reads as zeros, a length outside the table is clamped, and the status says so."""
    q, w, pages, table, lens = (t.cuda() for t in case([200, 90], h, 64, seed=10, fill=0))
    good = laga.paged_decode(q, w, pages, table, lens)[0]
    zeroed = torch.cat([pages, torch.zeros_like(pages[:1])])
    for page in (-1, pages.shape[0], 0x7fffffff, -2147483648):
        bad = table.clone()
        bad[0, 1] = page
        out, _, ws = laga.paged_decode(q, w, pages, bad, lens)
        assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK
        bad[0, 1] = pages.shape[0]
        # (zeros at a scale of 1 there, of 0 here: other references, so not bit for bit)
        assert rel_l2(out, f64(laga.paged_decode(q, w, zeroed, bad, lens)[0])) <= 5e-3 and torch.equal(out[1], good[1])
    out, _, ws = laga.paged_decode(q, w, pages, table, torch.tensor([-5, 90], dtype=torch.int32, device="cuda"))
    assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK and bool((out[0] == 0).all()) and torch.equal(out[1], good[1])
    out, _, ws = laga.paged_decode(q, w, pages, torch.zeros_like(table), torch.tensor([1 << 30, 90], dtype=torch.int32, device="cuda"))
    assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK


def test_results_repeat_and_do_not_depend_on_the_workspace(laga):  # noqa: F811
    q, w, pages, table, lens = (t.cuda() for t in case([3000, 10, 777], 32, 64, seed=11))
    a, _, ws = laga.paged_decode(q, w, pages, table, lens)
    ws.fill_(0xff)
    b = laga.paged_decode(q, w, pages, table, lens, workspace=ws)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = laga.paged_decode(q, w, pages, table, lens, stream=side)[0]
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def test_captured_and_replayed_with_other_lengths(laga):  # noqa: F811
    q, w, pages, table, lens = (t.cuda() for t in case([500, 300, 64], 16, 64, seed=12, fill=0))
    out, ws = torch.empty(3, 16, 128, dtype=BF16, device="cuda"), laga.alloc_workspace(laga.paged_decode_workspace_bytes(3, 16, cache8=True))
    laga.paged_decode(q, w, pages, table, lens, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        laga.paged_decode(q, w, pages, table, lens, out=out, workspace=ws)
    for new in ([500, 300, 64], [1, 0, 2], [333, 299, 17]):
        lens.copy_(torch.tensor(new, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(sum(new))).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, laga.paged_decode(q, w, pages, table, lens)[0])
        laga.check_status(ws)


def test_refusals(laga):  # noqa: F811
    q, w, pages, table, lens = (t.cuda() for t in case([64, 20], 16, 16, seed=13, fill=0))
    with pytest.raises(laga.LagaError) as err:               # a workspace for another form
        laga.paged_decode(q, w, pages, table, lens, workspace=laga.alloc_workspace(laga.paged_decode_workspace_bytes(2, 16, cache8=True) - 1024))
    assert err.value.code == laga.ERR_WORKSPACE_TOO_SMALL
    for bad in (pages[:, :-1], pages.view(-1), pages.view(torch.int8), pages.cpu()):
        with pytest.raises(ValueError):
            laga.paged_decode(q, w, bad, table, lens)
    with pytest.raises(laga.LagaError):
        laga.paged_decode(q, w, pages[:, : 8 * 644].contiguous(), table, lens)
    with pytest.raises(laga.LagaError):
        laga.paged_decode(q[..., :160].contiguous(), w[:, : 16 * 224].contiguous(), pages, table, lens)
    out, _, ws = laga.paged_decode(q[:0], w, pages, table[:0], lens[:0])
    assert out.shape == (0, 16, 128) and laga.query_status(ws)[0] == laga.OK
