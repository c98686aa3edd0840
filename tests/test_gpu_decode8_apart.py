"""One-token attention over the cache in 8 bits where a few tokens' weights stand far above their neighbours': tokens with a large key, a high score and
next to no value, as they are found at the start of a context.  What comes out is what the others leave, so it shows how exactly those are held."""
import pytest
import torch

import cache8_reference as c8
from parity import f64, rel_l2
from test_gpu_decode import BF16, laga  # noqa: F401  (laga: the fixture)
from test_gpu_decode8 import case, run
from test_gpu_decode8 import check as check_all

pytestmark = pytest.mark.gpu

# The four roundings of test_gpu_decode8.check, 4.5e-3; and of what is left beside a weight that stands only just not apart, 2^11 above the largest of the rest (over
# 32 heads 2^10), where that is at 2^-7 (2^-3) and each is off by 2^-15 (2^-10) at most: 2^-8 (2^-7) of the largest, over sqrt(3) in the mean square, and of the
# rest's mean square, which is at least 0.8 of their largest here: 2.8e-3 (5.6e-3).  Together 7.2e-3.
LIMIT = 7.5e-3


def check(tensors, out, lse):
    """Every request for itself: one without such a token has results thousands of times larger."""
    check_all(tensors, out, lse, l2=LIMIT)
    want = c8.decode(*tensors, 192 ** -0.5)[0]
    off = {b: rel_l2(out[b], want[b]) for b in range(len(want)) if tensors[4][b] > 1}
    assert max(off.values()) <= LIMIT, {b: (int(tensors[4][b]), e) for b, e in off.items() if e > LIMIT}


def sinks(lens, h, page, at, above, size, seed, mean=0.0, of=None):
    """Requests whose tokens `at` score `above` nats (a number, or one a token) higher than all others, whose scores are of order one; `size` is what
    the query has in the channel that says so, so a large one makes the tokens' keys, and with them their scales, small.  Values: normal, plus `mean`;
    of the tokens `at`, next to nothing.  q_nope is zero, so the scores come from the key alone."""
    above = [above] * len(at) if isinstance(above, (int, float)) else above

    def rows_of(b, rows):
        rows[:, :512] = rows[:, :512] * 0.25 + mean
        rows[:, 512:] *= 0.25
        rows[:, 512] = 0.0
        if of is None or b in of:
            for t, s in zip(at, above):
                if t < len(rows):
                    rows[t, 512] = s * 192 ** 0.5 / size
                    rows[t, :512] = 1e-3
        return rows

    q, w, pages, table, n = case(lens, h, page, seed=seed, fill=0xff, rows_of=rows_of)
    q[..., :128] = 0
    q[..., 128] = size
    return q, w, pages, table, n


@pytest.mark.parametrize("h", [16, 24, 32, 33, 64, 130])
@pytest.mark.parametrize("above,size", [(5.0, 1.0), (9.0, 1.0), (13.0, 1.0), (9.0, 16.0), (13.0, 16.0), (20.0, 4.0)])
def test_a_first_token_that_stands_apart(laga, h, above, size):  # noqa: F811
    tensors = sinks([100, 700, 33, 128, 0, 2, 64, 129], h, 64, [0], above, size, seed=90)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("h", [5, 32, 64])
@pytest.mark.parametrize("at", [[0, 1], [0, 31, 70, 99], [3, 5, 9, 31, 64, 95, 200], [127], [130, 500], [0, 129, 257, 385], [0, 31, 64, 1000, 1001, 1088, 1091]])
def test_places_of_those_that_stand_apart(laga, h, at):  # noqa: F811
    """Up to four of 32 neighbours, half of the runs of 32 in any tile without one; in one tile and in several, in pages of 16."""
    tensors = sinks([1100, 140], h, 16, at, [12.0 + 0.5 * (i % 3) for i in range(len(at))], 1.0, seed=91)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("at", [[0, 7, 150], [0, 1, 70, 75], [2, 3, 30, 31]])
@pytest.mark.parametrize("h,B", [(16, 150), (16, 420), (32, 210), (64, 130)])
def test_among_many_requests(laga, h, B, at):  # noqa: F811
    """A CTA goes through many of them, with and without such tokens; whichever kernel joins the pieces."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 300, (B,), generator=g).tolist()
    lens[B // 3] = 4000
    tensors = sinks(lens, h, 32, at, 11.0, 2.0, seed=92, of=set(range(0, B, 2)) | {B // 3})
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("h", [16, 64])
@pytest.mark.parametrize("steps", [(8.0, 16.0, 24.0), (24.0, 16.0, 8.0), (10.0, 60.0, 10.0), (10.0, 10.0, 60.0)])
def test_one_above_another(laga, h, steps):  # noqa: F811
    """In one tile and in two, the later above the earlier and below; 60 nats are more than the 2^40 by which the reference may lie below."""
    tensors = sinks([150] * 160, h, 32, [10, 70, 140], list(steps), 8.0, seed=93)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("h", [16, 32, 64])
def test_more_of_them_than_there_are_places(laga, h):  # noqa: F811
    """Forty of them in a piece: those past the places set the reference.  Their values are like the others' here, so what they drown is nothing."""
    def rows_of(b, rows):
        rows[:, 512:] *= 0.25
        rows[:, 512] = 0.0
        rows[3::7, 512] = 9.0 * 192 ** 0.5 / 8.0
        return rows

    q, w, pages, table, n = case([280, 281], h, 64, seed=94, rows_of=rows_of)
    q[..., :128] = 0
    q[..., 128] = 8.0
    tensors = (q, w, pages, table, n)
    check(tensors, *run(laga, tensors))


def test_repeats_and_replays(laga):  # noqa: F811
    """The same bits again, over a workspace that holds anything, and from a graph after other requests went through it."""
    for h in (16, 32, 64):
        q, w, pages, table, n = (t.cuda() for t in sinks([600, 90, 33, 300] * 12, h, 32, [0, 5, 40], 12.0, 1.0, seed=95))
        a, _, ws = laga.paged_decode(q, w, pages, table, n)
        for fill in (0xff, 0x00, 0x5a):
            ws.fill_(fill)
            assert torch.equal(a, laga.paged_decode(q, w, pages, table, n, workspace=ws)[0])
        out = torch.empty_like(a)
        laga.paged_decode(q, w, pages, table, n, out=out, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            laga.paged_decode(q, w, pages, table, n, out=out, workspace=ws)
        held = n.clone()
        for lens in (held // 2, held.flip(0).clamp(max=90), held):
            n.copy_(torch.minimum(lens, held))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, laga.paged_decode(q, w, pages, table, n)[0])
        assert torch.equal(out, a)


def test_not_finite_beside_one_that_stands_apart(laga):  # noqa: F811
    for h in (16, 64):
        q, w, pages, table, n = sinks([100, 130, 64, 300], h, 16, [0, 20], 12.0, 1.0, seed=96)
        clean, _ = run(laga, (q, w, pages, table, n))
        codes, scales = c8.planes(pages)
        codes[int(table[0, 0]), 3, 7] = 0x7f
        scales[int(table[1, 3]), 5] = float("nan")
        q[3, 0, 130] = float("inf")
        out, lse = run(laga, (q, w, pages, table, n))
        assert bool(torch.isnan(out[:2].float()).all()) and bool(torch.isnan(lse[:2]).all()) and bool(torch.isnan(out[3, 0].float()).all())
        assert torch.equal(out[3, 1:], clean[3, 1:]) and torch.equal(out[2], clean[2])


def test_bad_pages_beside_one_that_stands_apart(laga):  # noqa: F811
    """A page outside the cache reads as zeros (whose scores stand apart of scores far below); the status says so, the others' results stay."""
    for h in (16, 64):
        tensors = sinks([200, 90], h, 64, [0, 100], 12.0, 1.0, seed=97)
        q, w, pages, table, n = (t.cuda() for t in tensors)
        good = laga.paged_decode(q, w, pages, table, n)[0]
        zeroed = torch.cat([pages, torch.zeros_like(pages[:1])])
        for page in (-1, 0x7fffffff):
            bad = table.clone()
            bad[0, 1] = page
            out, _, ws = laga.paged_decode(q, w, pages, bad, n)
            assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK
            bad[0, 1] = pages.shape[0]
            assert rel_l2(out, f64(laga.paged_decode(q, w, zeroed, bad, n)[0])) <= 5e-3 and torch.equal(out[1], good[1])
