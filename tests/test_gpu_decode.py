"""One-token attention over the paged latent cache on the GPU against the explicit form in float64."""
import math

import pytest
import torch

import serving_reference as ref
from parity import f64, rel_l2

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def laga():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_17644_b200 import laga as _laga
    _laga.lib()
    return _laga


def case(lens, h, page, seed=0, columns=None, spare=2, fill=float("nan")):
    """Pages in random order; everything no token owns (rows behind the last token, spare pages) holds `fill`, and the table's
    unused columns hold nonsense."""
    g = torch.Generator().manual_seed(seed + sum(lens) + h)
    held = [-(-t // page) for t in lens]
    columns = max(1, max(held)) if columns is None else columns
    n_pages = sum(held) + spare
    perm = torch.randperm(n_pages, generator=g).to(torch.int32).tolist()
    cache = torch.full((n_pages, page, 576), fill, dtype=BF16)
    table = torch.full((len(lens), columns), 0x7fffffff, dtype=torch.int32)
    for b, t in enumerate(lens):
        mine = [perm.pop() for _ in range(held[b])]
        if mine:
            table[b, : held[b]] = torch.tensor(mine, dtype=torch.int32)
            rows = torch.randn(t, 576, generator=g).to(BF16)
            for k, p in enumerate(mine):
                part = rows[k * page:(k + 1) * page]
                cache[p, : len(part)] = part
    q = torch.randn(len(lens), h, 192, generator=g).to(BF16)
    w = (torch.randn(512, h * 256, generator=g) * 512 ** -0.5).to(BF16)
    return q, w, cache, table, torch.tensor(lens, dtype=torch.int32)


def run(laga, tensors, scale=None):
    dev = [t.cuda() for t in tensors]
    B, h = tensors[0].shape[:2]
    out = torch.full((B, h, 128), float("nan"), dtype=BF16, device="cuda")
    lse = torch.full((B, h), float("nan"), device="cuda")
    _, _, ws = laga.paged_decode(*dev, softmax_scale=scale, out=out, lse=lse)
    laga.check_status(ws, where="laga_paged_decode")
    return out, lse


def check(tensors, out, lse, scale=192 ** -0.5, l2=5e-3):
    want, want_lse, b_out, b_lse = ref.decode(*tensors, scale)
    assert not torch.isnan(f64(out)).any()
    err = (f64(out) - want).abs()
    assert float((err - b_out).max()) <= 0, (float(err.max()), float(b_out.max()))
    # four independent roundings to bf16, each at most U / sqrt(3) in the mean square of its relative error: 2 U / sqrt(3) = 4.5e-3
    if float(want.norm()) > 0:
        assert rel_l2(out, want) <= l2
    live = tensors[4] > 0
    assert bool((lse[~live].cpu() == -math.inf).all()) and bool((out[~live] == 0).all())
    assert float(((f64(lse) - want_lse)[live].abs() - b_lse[live]).max()) <= 0 if bool(live.any()) else True


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("h", [1, 16, 40])
def test_lengths_around_every_boundary(laga, h, page):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 0, 31, 33, 200, 257]
    tensors = case(lens, h, page)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("B,h", [(1, 16), (1, 128), (3, 5), (5, 24), (2, 33), (2, 64), (2, 65), (1, 200), (150, 16), (300, 2)])
def test_batches_and_heads(laga, B, h):
    g = torch.Generator().manual_seed(B * 7 + h)
    lens = torch.randint(0, 700 if B < 10 else 90, (B,), generator=g).tolist()
    tensors = case(lens, h, 64, seed=1)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("B,h", [(17, 128), (34, 128), (45, 64), (129, 33), (300, 16)])
def test_several_request_tiles_per_head(laga, B, h):
    """More tiles of 16 requests than CTAs for a head: the joining kernel's pipeline, with last tiles of 1, 2, 12 and 13 requests."""
    g = torch.Generator().manual_seed(B + h)
    lens = torch.randint(0, 70, (B,), generator=g).tolist()
    lens[-1] = 1500                                     # one request in many pieces, in the last tile
    tensors = case(lens, h, 32, seed=10)
    check(tensors, *run(laga, tensors))


@pytest.mark.parametrize("lens,h,page", [([511], 16, 32), ([9001], 16, 64), ([20011, 3], 4, 16), ([12345, 1, 0, 6000], 64, 64), ([15000, 777], 128, 256)])
def test_long_contexts(laga, lens, h, page):
    tensors = case(lens, h, page, seed=2)
    check(tensors, *run(laga, tensors))


def test_all_empty_and_one_token(laga):
    tensors = case([0, 0, 0], 16, 64)
    check(tensors, *run(laga, tensors))
    tensors = case([1], 16, 16)
    out, lse = run(laga, tensors)
    check(tensors, out, lse)
    v = tensors[2][tensors[3][0, 0], 0, :512].double() @ tensors[1].double().view(512, 16, 256)[..., 128:].reshape(512, -1)
    assert rel_l2(out.reshape(1, -1), v) <= 2 * ref.U                 # softmax of one score is 1: the value itself


def test_growing_scores_move_the_maximum(laga):
    """Scores that grow along the context (the running maximum moves in every tile, by far more than 2^8), fall, and alternate
    in sign: the rescaling of the accumulator."""
    for shape in ("up", "down", "alternate"):
        q, w, cache, table, lens = case([1500, 900], 16, 64, seed=3, fill=0.0)
        ramp = {"up": torch.linspace(0.1, 30, 1536), "down": torch.linspace(30, 0.1, 1536), "alternate": torch.tensor([30.0, -30.0]).repeat(768)}[shape]
        for b in range(2):
            t = int(lens[b])
            for k in range(-(-t // 64)):
                n = min(64, t - 64 * k)
                p = int(table[b, k])
                direction = q[b, 0, 128:].float().sign()
                cache[p, :n, 512:] = (direction * ramp[64 * k: 64 * k + n, None]).to(BF16)
        tensors = (q, w, cache, table, lens)
        check(tensors, *run(laga, tensors))


def test_values_that_are_not_finite(laga):
    """NaN and infinity in a request's own tokens reach its result; nothing reaches another request's."""
    tensors = case([100, 130, 64], 16, 16, seed=4)
    q, w, cache, table, lens = tensors
    clean, _ = run(laga, tensors)
    cache[int(table[1, 3]), 5, 100] = float("nan")
    cache[int(table[0, 0]), 0, 7] = float("inf")
    out, lse = run(laga, tensors)
    assert bool(torch.isnan(out[1].float()).all()) and bool(torch.isnan(lse[1]).all())
    assert not bool(torch.isfinite(out[0].float()).all())
    assert torch.equal(out[2], clean[2])


def test_keys_of_minus_infinity(laga):
    """Tokens taken out by a key of minus infinity weigh nothing, also where they fill a tile, or all that one CTA has of the
    request: the result is that of the other tokens alone."""
    lens = [20000, 100]
    q, w, cache, table, lens = case(lens, 4, 16, seed=9, fill=0.0)
    q[..., 128 + 3] = q[..., 128 + 3].abs().clamp_min(0.125)
    rows = cache[table[0].long()].reshape(-1, 576)[:20000]
    at = torch.arange(20000)
    out_of = (at < 2048) | ((at // 64) % 2 == 0) | (at % 64 == 11) | (at >= 19000)
    rows[out_of, 512 + 3] = -math.inf
    cache[table[0].long()] = rows.view(-1, 16, 576)
    kept = cache.clone()
    left = rows[~out_of]
    n = -(-len(left) // 16)
    kept[table[0, :n].long()] = torch.nn.functional.pad(left, (0, 0, 0, 16 * n - len(left))).view(-1, 16, 576)
    out, lse = run(laga, (q, w, cache, table, lens))
    check((q, w, kept, table, torch.tensor([len(left), 100], dtype=torch.int32)), out, lse)


def test_shared_pages_and_repeated_requests(laga):
    """Prefix sharing: two requests over the same pages, different lengths, and the same request three times."""
    q, w, cache, table, lens = case([400], 16, 32, seed=5)
    q = torch.cat([q, torch.randn_like(q.float()).to(BF16), q, q])
    table = table.expand(4, -1).contiguous()
    lens = torch.tensor([400, 333, 400, 400], dtype=torch.int32)
    tensors = (q, w, cache, table, lens)
    out, lse = run(laga, tensors)
    check(tensors, out, lse)


def test_bad_pages_and_lengths_are_reported(laga):
    """Bad entries are bounds-checked in the kernel: a page number outside the cache reads as zeros, a length outside the table
    is clamped, and the status says so."""
    q, w, cache, table, lens = (t.cuda() for t in case([200, 90], 16, 64, seed=6, fill=0.0))
    good = laga.paged_decode(q, w, cache, table, lens)[0]
    for page in (-1, cache.shape[0], 0x7fffffff, -2147483648):
        bad = table.clone()
        bad[0, 1] = page
        out, _, ws = laga.paged_decode(q, w, cache, bad, lens)
        assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK
        zeroed = torch.cat([cache, torch.zeros_like(cache[:1])])
        bad[0, 1] = cache.shape[0]
        assert torch.equal(out, laga.paged_decode(q, w, zeroed, bad, lens)[0]) and torch.equal(out[1], good[1])
    out, _, ws = laga.paged_decode(q, w, cache, table, torch.tensor([-5, 90], dtype=torch.int32, device="cuda"))
    assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK and bool((out[0] == 0).all()) and torch.equal(out[1], good[1])
    full = torch.zeros_like(table)
    out, _, ws = laga.paged_decode(q, w, cache, full, torch.tensor([1 << 30, 90], dtype=torch.int32, device="cuda"))
    assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK
    assert torch.equal(out, laga.paged_decode(q, w, cache, full, torch.tensor([256, 90], dtype=torch.int32, device="cuda"))[0])


def test_results_repeat_and_do_not_depend_on_the_workspace(laga):
    q, w, cache, table, lens = (t.cuda() for t in case([3000, 10, 777], 32, 64, seed=7))
    a, _, ws = laga.paged_decode(q, w, cache, table, lens)
    ws.fill_(0xff)
    b = laga.paged_decode(q, w, cache, table, lens, workspace=ws)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = laga.paged_decode(q, w, cache, table, lens, stream=side)[0]
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def test_what_a_side_stream_writes_comes_from_its_pool(laga):
    """The current stream must not get the output or the workspace back while the side stream may still be at work."""
    q, w, cache, table, lens = (t.cuda() for t in case([300, 20], 16, 64, seed=11))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, _, ws = laga.paged_decode(q, w, cache, table, lens, stream=side)
    mine = {out.untyped_storage().data_ptr(), ws.untyped_storage().data_ptr()}
    n_out, n_ws = out.numel(), ws.numel()
    del out, ws
    again = [torch.empty(n_out, dtype=BF16, device="cuda"), laga.alloc_workspace(n_ws)]
    assert not mine & {t.untyped_storage().data_ptr() for t in again}
    torch.cuda.synchronize()


def test_captured_and_replayed_with_other_lengths(laga):
    """One captured call serves every step: lengths, table and queries are read when it is replayed."""
    q, w, cache, table, lens = (t.cuda() for t in case([500, 300, 64], 16, 64, seed=8, fill=0.0))
    out, ws = torch.empty(3, 16, 128, dtype=BF16, device="cuda"), laga.alloc_workspace(laga.paged_decode_workspace_bytes(3, 16))
    laga.paged_decode(q, w, cache, table, lens, out=out, workspace=ws)          # warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        laga.paged_decode(q, w, cache, table, lens, out=out, workspace=ws)
    for new in ([500, 300, 64], [1, 0, 2], [333, 299, 17]):
        lens.copy_(torch.tensor(new, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(sum(new))).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, laga.paged_decode(q, w, cache, table, lens)[0])
        laga.check_status(ws)
