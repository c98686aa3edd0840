"""The rotary block in service over a latent cache in 8 bits: prompts and decode steps against the same rows attended to densely, captured steps,
refused ones, and requests read back."""
import pytest
import torch

import cache8_reference as c8
from parity import rel_l2
from test_gpu_serving import BF16, make_block, pkg  # noqa: F401  (pkg: the fixture)

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def dense(pkg, blk, hidden):  # noqa: F811
    """One sequence through the block's own steps, with its latents and keys as a cache in 8 bits holds them."""
    laga = pkg.laga
    n = len(hidden)
    pos, slots = blk.positions(n), torch.arange(n, **I32)
    q = laga.rope(laga.linear(hidden, blk.w_q)[0].view(n, blk.n_heads, 192), pos, blk.rope)
    pages = laga.cache_append(laga.linear(hidden, blk.w_kv_a)[0], blk.ln_gamma, blk.ln_beta, pos, blk.rope, slots, c8.empty_pages(-(-n // 16), 16).cuda(), blk.eps)
    latent, k_pe = laga.cache_read(pages, slots)
    out = laga.fwd(q, latent, k_pe, blk.w_kv_b, softmax_scale=blk.softmax_scale)[0]
    return laga.linear(out.view(n, -1), blk.w_o)[0]


@torch.no_grad()
@pytest.mark.parametrize("heads,page", [(16, 16), (40, 64)])
def test_prompts_and_decode_steps_against_one_pass(pkg, heads, page):  # noqa: F811
    """Three requests, prompts of 70, 1 and 129 tokens, then 20 decode steps (crossing pages).  Prompts: the same kernels on the same rows.  Decode: 2e-2,
    as the bf16 cache's (the absorbed form's few roundings of at most 2^-8 against the explicit form's)."""
    laga = pkg.laga
    blk = make_block(pkg, heads=heads)
    prompts, steps = [70, 1, 129], 20
    g = torch.Generator().manual_seed(5)
    seqs = [torch.randn(n + steps, 512, generator=g).to(BF16).cuda() for n in prompts]
    cache = pkg.LatentCache(n_pages=-(-24 * 16 // page) + 3, n_requests=3, max_tokens=160, page_size=page, n_layers=2, bits=8)
    pages = cache.pages[1]
    cu = [0, 70, 71, 200]
    step = cache.plan(torch.tensor(prompts, **I32), 200)
    laga.check_status(step.status)
    y = blk.prefill(torch.cat([s[:n] for s, n in zip(seqs, prompts)]), pages, step, cu)
    laga.check_status(step.status)
    decoded = []
    ws = laga.alloc_workspace(laga.paged_decode_workspace_bytes(3, heads, cache8=True))
    for i in range(steps):
        step = cache.plan(torch.ones(3, **I32), 3)
        decoded.append(blk.decode(torch.stack([s[n + i] for s, n in zip(seqs, prompts)]), pages, step, cache.block_table, workspace=ws))
        laga.check_status(ws)
    assert not bool(cache.pages[0].any())
    for b, n in enumerate(prompts):
        whole = dense(pkg, blk, seqs[b])
        assert rel_l2(y[cu[b]:cu[b + 1]], whole[:n]) <= 1e-6
        assert rel_l2(torch.stack([d[b] for d in decoded]), whole[n:]) <= 2e-2
        latent, k_pe = cache.read(b, n + steps + 3, layer=1)
        assert not bool(latent[n + steps:].any()) and not bool(k_pe[n + steps:].any())
        again = pkg.LatentCache(n_pages=24, n_requests=1, max_tokens=160, page_size=16)
        hold = again.plan(torch.tensor([n + steps], **I32), n + steps)
        rows = torch.cat([latent, k_pe], 1)[: n + steps]
        again.pages[0].view(-1, 576)[hold.slots.long()] = rows                 # moved to a cache in bf16, and read back from there
        l2, k2 = again.read(0, n + steps)
        assert torch.equal(l2, latent[: n + steps]) and torch.equal(k2, k_pe[: n + steps])


def test_rounding_of_the_cache_is_what_8_bits_cost(pkg):  # noqa: F811
    """The block over 8 bits against the block over 16: what differs is the cache's rounding.  A latent channel is off by at most 2^-4, in the mean
    square (uniform in its step, spread over the binade) about 2^-4 / sqrt(3) * 0.72 = 2.6e-2; a value is a sum of 512 of them with independent errors, so
    off by as much of itself; an output is a mean of values, whose errors are independent too: no more than that, with the scores' part beside it."""
    blk = make_block(pkg, heads=16)
    x = torch.randn(300, 512, generator=torch.Generator().manual_seed(8)).to(BF16).cuda()
    outs = []
    for bits in (8, 16):
        cache = pkg.LatentCache(n_pages=20, n_requests=1, max_tokens=320, page_size=16, bits=bits)
        outs.append(blk.prefill(x, cache.pages[0], cache.plan(torch.tensor([300], **I32), 300), [0, 300]))
    assert 1e-3 <= rel_l2(outs[0], outs[1]) <= 2 * 2.6e-2


def test_captured_decode_steps_equal_eager_ones(pkg):  # noqa: F811
    laga = pkg.laga
    blk = make_block(pkg, heads=16)
    g = torch.Generator().manual_seed(6)
    x = torch.randn(6, 4, 512, generator=g).to(BF16).cuda()

    def service():
        cache = pkg.LatentCache(n_pages=16, n_requests=4, max_tokens=64, page_size=16, bits=8)
        prompt = torch.randn(49, 512, generator=torch.Generator().manual_seed(7)).to(BF16).cuda()
        blk.prefill(prompt, cache.pages[0], cache.plan(torch.tensor([14, 0, 30, 5], **I32), 49), [0, 14, 14, 44, 49])
        return cache

    one = torch.ones(4, **I32)
    eager_cache, cache = service(), service()
    ws = laga.alloc_workspace(laga.paged_decode_workspace_bytes(4, 16, cache8=True))
    eager = [blk.decode(x[i], eager_cache.pages[0], eager_cache.plan(one, 4), eager_cache.block_table) for i in range(6)]
    static = torch.empty_like(x[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = blk.decode(static, cache.pages[0], cache.plan(one, 4), cache.block_table, workspace=ws)
    for i in range(6):
        static.copy_(x[i])
        graph.replay()
        assert torch.equal(y, eager[i]), i
    assert torch.equal(cache.pages[0], eager_cache.pages[0])


def test_refused_prompts_and_padding(pkg):  # noqa: F811
    """A step that is not one of new prompts leaves the cache as it was, gives NaN and says so; rows without a slot are padding."""
    laga = pkg.laga
    blk = make_block(pkg, heads=16)
    x = torch.randn(64, 512, generator=torch.Generator().manual_seed(9)).to(BF16).cuda()
    cache = pkg.LatentCache(n_pages=8, n_requests=2, max_tokens=64, page_size=16, bits=8)
    step = cache.plan(torch.tensor([20, 12], **I32), 40)
    y = blk.prefill(x[:40], cache.pages[0], step, [0, 20, 32, 40])         # eight rows of padding as a sequence of their own
    laga.check_status(step.status)
    assert bool(y[:32].isfinite().all())
    before = cache.pages[0].clone()
    step = cache.plan(torch.tensor([4, 4], **I32), 8)                        # requests that hold tokens already
    bad = blk.prefill(x[:8], cache.pages[0], step, [0, 4, 8])
    assert bool(bad.isnan().all()) and torch.equal(cache.pages[0], before)
    with pytest.raises(laga.LagaError) as err:
        laga.check_status(step.status)
    assert err.value.code == laga.ERR_CACHE_PLAN


def test_decode_step_for_some_of_the_requests(pkg):  # noqa: F811
    blk = make_block(pkg, heads=16)
    g = torch.Generator().manual_seed(12)
    lens = [40, 25, 33]
    prompts = [torch.randn(n, 512, generator=g).to(BF16).cuda() for n in lens]
    token = torch.randn(4, 512, generator=g).to(BF16).cuda()
    cache = pkg.LatentCache(n_pages=12, n_requests=3, max_tokens=64, page_size=16, bits=8)
    blk.prefill(torch.cat(prompts), cache.pages[0], cache.plan(torch.tensor(lens, **I32), 98), [0, 40, 65, 98])
    before = cache.pages[0].clone()
    step = cache.plan(torch.tensor([1, 0, 1], **I32), 4)
    y = blk.decode(token, cache.pages[0], step, cache.block_table, requests=torch.tensor([0, 2, 2, 2], device="cuda"))
    codes, was = (c8.planes(p.cpu())[0].reshape(-1, 640) for p in (cache.pages[0], before))
    assert sorted((codes != was).any(-1).nonzero().view(-1).tolist()) == sorted(step.slots[:2].tolist())
    with torch.no_grad():
        for row, b in enumerate((0, 2)):
            assert rel_l2(y[row], dense(pkg, blk, torch.cat([prompts[b], token[row:row + 1]]))[-1]) <= 2e-2
