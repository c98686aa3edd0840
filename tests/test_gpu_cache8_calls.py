"""The 8-bit cache's calls as a service makes them: from two threads at once, in two graphs over one workspace, into results that begin on any
16-byte boundary, over caches of more than 2^32 bytes, with a workspace for more requests than there are."""
import threading

import pytest
import torch

import cache8_reference as c8
from test_gpu_cache8 import inputs
from test_gpu_decode import BF16, laga  # noqa: F401  (laga: the fixture)
from test_gpu_decode8 import case, check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def test_calls_from_two_threads(laga):  # noqa: F811
    """Each thread on a stream of its own with tensors of its own; the second's requests take the kernels for many."""
    def work(seed, lens, h, rounds):
        q, w, pages, table, n = (t.cuda() for t in case(lens, h, 16, seed=seed, fill=0))
        kv, gamma, beta, _ = (None if t is None else t.cuda() for t in inputs(len(lens), seed))
        rope, slots, pos = laga.rope_plan(64), table[:, 0] * 16, (n - 1).clamp(min=0)      # each request's first row anew
        slots = torch.where(n > 0, slots, -1).to(torch.int32)
        out = []
        for _ in range(rounds):
            cache = laga.cache_append(kv, gamma, beta, pos, rope, slots, pages.clone())
            latent, k_pe = laga.cache_read(cache, slots)
            y, _, ws = laga.paged_decode(q, w, cache, table, n)
            out.append((cache, latent, k_pe, y, ws[:4].clone()))
        return out

    jobs = [(71, [300, 0, 17, 900], 16, 40), (72, [40, 3, 0] * 47, 64, 40)]
    alone = [work(*job[:3], 1)[0] for job in jobs]
    torch.cuda.synchronize()
    results, errors, gate = [None, None], [], threading.Barrier(2)

    def thread(k):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                gate.wait(60)
                results[k] = work(*jobs[k])
            stream.synchronize()
        except BaseException as e:  # noqa: BLE001  (shown by the assertion below)
            errors.append(e)

    threads = [threading.Thread(target=thread, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not errors and not any(t.is_alive() for t in threads), errors
    for k in range(2):
        assert len(results[k]) == jobs[k][3]
        for got in results[k]:
            assert all(torch.equal(a, b) for a, b in zip(got, alone[k]))


def test_two_graphs_over_one_workspace(laga):  # noqa: F811
    """Steps of 140 and of 3 requests captured over the same workspace, made for the larger: replayed in turn, each gives its own results."""
    many = [t.cuda() for t in case([33] * 139 + [800], 64, 32, seed=73, fill=0)]
    few = [t.cuda() for t in case([700, 0, 65], 64, 32, seed=74, fill=0)]
    ws = laga.alloc_workspace(laga.paged_decode_workspace_bytes(140, 64, cache8=True))
    want = [laga.paged_decode(*t)[0] for t in (many, few)]
    outs = [torch.empty_like(w) for w in want]
    for t, o in zip((many, few), outs):
        laga.paged_decode(*t, out=o, workspace=ws)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in outs]
    for graph, t, o in zip(graphs, (many, few), outs):
        with torch.cuda.graph(graph):
            laga.paged_decode(*t, out=o, workspace=ws)
    for k in (0, 1, 1, 0, 1):
        outs[k].fill_(float("nan"))
        graphs[k].replay()
        assert torch.equal(outs[k], want[k])
        laga.check_status(ws)


def test_workspace_grows_with_the_requests(laga):  # noqa: F811
    for h in (1, 16, 33, 64, 128, 200):
        sizes = [laga.paged_decode_workspace_bytes(B, h, cache8=True) for B in range(1, 700)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("shift", [0, 8, 16, 24])
def test_results_on_any_sixteen_bytes(laga, shift):  # noqa: F811
    """Results (and the decode's) that begin 16, 32 and 48 bytes into an allocation, and a cache that begins 16 bytes into one."""
    M, page = 61, 16
    kv, gamma, beta, pos = (t.cuda() for t in inputs(M))
    slots = torch.randperm(5 * page, generator=torch.Generator().manual_seed(shift))[:M].to(torch.int32).cuda()
    room = torch.zeros(5 * page * 644 + 64, dtype=torch.uint8, device="cuda")
    pages = room[2 * shift: 2 * shift + 5 * page * 644].view(5, page * 644)
    laga.cache_append(kv, gamma, beta, pos, laga.rope_plan(64), slots, pages)
    want = laga.cache_read(pages.clone(), slots)
    held = [torch.full((M * n + 64,), 7.0, dtype=BF16, device="cuda") for n in (512, 64)]
    latent, k_pe = held[0][shift: shift + M * 512].view(M, 512), held[1][shift: shift + M * 64].view(M, 64)
    laga.cache_read(pages, slots, latent=latent, k_pe=k_pe)
    assert torch.equal(latent, want[0]) and torch.equal(k_pe, want[1])
    assert all(bool((t[:shift] == 7).all()) and bool((t[shift + M * n:] == 7).all()) for t, n in zip(held, (512, 64)))

    q, w, cache, table, n = (t.cuda() for t in case([100, 37], 20, 16, seed=75, fill=0))
    want = laga.paged_decode(q, w, cache, table, n)[0]
    room = torch.zeros(cache.numel() + 64, dtype=torch.uint8, device="cuda")
    moved = room[2 * shift: 2 * shift + cache.numel()].view(cache.shape)
    moved.copy_(cache)
    out = torch.full((q.numel() + 64,), 7.0, dtype=BF16, device="cuda")
    y = out[shift: shift + want.numel()].view(want.shape)
    laga.paged_decode(q, w, moved, table, n, out=y)
    assert torch.equal(y, want) and bool((out[:shift] == 7).all()) and bool((out[shift + want.numel():] == 7).all())


def test_decode_over_a_cache_of_five_gigabytes(laga):  # noqa: F811
    """Pages on both sides of 2^31 and 2^32 bytes."""
    page, n_pages = 64, 122_000
    size = page * 644
    cache = torch.empty(n_pages, size, dtype=torch.uint8, device="cuda")
    edges = [0, 2 ** 31 // size, 2 ** 32 // size, 2 ** 32 // size + 1, n_pages - 1, 110_001, 17]
    for h in (16, 64):
        q, w, pages, table, n = case([64 * len(edges), 100], h, page, seed=76, fill=0)
        far = table.clone()
        for k, p in enumerate(edges):
            cache[p] = pages[table[0, k]].cuda()
            far[0, k] = p
        far[1, :2] = torch.tensor([n_pages - 2, 2 ** 31 // size + 1])
        for k in range(2):
            cache[far[1, k]] = pages[table[1, k]].cuda()
        here, _, ws = laga.paged_decode(q.cuda(), w.cuda(), cache, far.cuda(), n.cuda())
        laga.check_status(ws)
        assert torch.equal(here, laga.paged_decode(q.cuda(), w.cuda(), pages.cuda(), table.cuda(), n.cuda())[0])


def test_pages_whose_tables_repeat(laga):  # noqa: F811
    """A table that names one page many times, within a request and across requests."""
    q, w, pages, table, n = case([64, 500, 37, 129], 24, 16, seed=77)
    table[1, :32] = table[0, :4].repeat(8)
    table[3, :9] = table[0, 1]
    tensors = (q, w, pages, table, n)
    check(tensors, *run(laga, tensors))


def test_heads_that_share_nothing_but_the_cache(laga):  # noqa: F811
    """The result of a head does not depend on the heads beside it, whatever their number and place."""
    q, w, pages, table, n = (t.cuda() for t in case([300, 64, 1], 64, 32, seed=78, fill=0))
    whole = laga.paged_decode(q, w, pages, table, n)[0]
    for first, h in ((0, 64), (5, 16), (40, 24), (63, 1)):
        part = laga.paged_decode(q[:, first: first + h].contiguous(), w.view(512, 64, 256)[:, first: first + h].reshape(512, -1).contiguous(), pages, table, n)[0]
        # (up to 32 heads a CTA the weights' parts are others: two of 2^-8 and the result's rounding apart)
        assert float((part.float() - whole[:, first: first + h].float()).norm() / whole[:, first: first + h].float().norm()) <= 8e-3


def test_lengths_past_the_table_are_clamped_for_many_requests_too(laga):  # noqa: F811
    q, w, pages, table, n = (t.cuda() for t in case([20] * 140, 64, 16, seed=79, fill=0))
    good = laga.paged_decode(q, w, pages, table, n)[0]
    n[3], n[139] = -7, 1 << 30
    full = n.clone()
    full[3], full[139] = 0, table.shape[1] * 16
    table[139, :] = table[138, 0]
    want = laga.paged_decode(q, w, pages, table, full)[0]
    out, _, ws = laga.paged_decode(q, w, pages, table, n)
    assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK
    assert torch.equal(out, want) and bool((out[3] == 0).all()) and torch.equal(out[4:138], good[4:138])


def test_reads_of_repeated_slots(laga):  # noqa: F811
    pages = c8.empty_pages(3, 32, 0).cuda()
    kv, gamma, beta, pos = (t.cuda() for t in inputs(96))
    laga.cache_append(kv, gamma, beta, pos, laga.rope_plan(64), torch.arange(96, dtype=torch.int32, device="cuda"), pages)
    all_of_them = laga.cache_read(pages, torch.arange(96, dtype=torch.int32, device="cuda"))
    slots = torch.tensor([5, 5, 95, -1, 96, 0, 5, -2147483648, 2147483647], dtype=torch.int32, device="cuda")
    for got, rows in zip(laga.cache_read(pages, slots), all_of_them):
        want = rows[slots.long().clamp(0, 95)].masked_fill(((slots < 0) | (slots > 95))[:, None], 0)
        assert torch.equal(got, want)


@pytest.mark.parametrize("h", [5, 16, 32, 64])
def test_a_million_tokens(laga, h):  # noqa: F811
    """A page named 1024 times weighs its tokens 1024 times: the result of the page alone, and a log-sum-exp larger by ln 1024."""
    q, w, pages, table, n = (t.cuda() for t in case([1024, 1024], h, 1024, seed=80, fill=0))
    once, lse = torch.empty(2, h, 128, dtype=BF16, device="cuda"), torch.empty(2, h, device="cuda")
    laga.paged_decode(q, w, pages, table, n, out=once, lse=lse)
    far, far_lse = torch.empty_like(once), torch.empty_like(lse)
    _, _, ws = laga.paged_decode(q, w, pages, table.repeat(1, 1024).contiguous(), n * 1024, out=far, lse=far_lse)
    laga.check_status(ws)
    # weights' parts, the joined latent's and the result's roundings, 2^-8 each, on both sides
    assert float((far.float() - once.float()).norm() / once.float().norm()) <= 8e-3
    # the sums differ by their weights' roundings, 2^-8 at most and of either sign
    assert float((far_lse - lse - 6.931471805599453).abs().max()) <= 2.0 ** -7


def test_twenty_thousand_requests(laga):  # noqa: F811
    """Against the same requests in calls of 40, whose lines and kernels are others."""
    B, h, page = 20_000, 2, 16
    g = torch.Generator().manual_seed(81)
    lens = torch.randint(0, 50, (B,), generator=g, dtype=torch.int32)
    base = case([16] * 400, h, page, seed=82, fill=0)
    pages, w = base[2].cuda(), base[1].cuda()
    q = torch.randn(B, h, 192, generator=g).to(BF16).cuda()
    table = torch.randint(0, 400, (B, 4), generator=g, dtype=torch.int32)
    table = base[3][:, 0][table.long()].to(torch.int32).contiguous().cuda()      # pages that hold tokens
    lens = lens.cuda()
    out, _, ws = laga.paged_decode(q, w, pages, table, lens)
    laga.check_status(ws)
    assert bool((out[lens == 0] == 0).all()) and not bool(torch.isnan(out.float()).any())
    for first in (0, 7_960, 19_960):
        at = slice(first, first + 40)
        part = laga.paged_decode(q[at], w, pages, table[at], lens[at])[0].float()
        assert float((out[at].float() - part).norm() / part.norm()) <= 8e-3
