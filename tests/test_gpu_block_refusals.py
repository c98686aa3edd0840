"""Steps that are not what the block's prefill and decode are for are refused on the device, not answered wrongly."""
import pytest
import torch

from parity import rel_l2
from test_gpu_serving import BF16, make_block, pkg  # noqa: F401  (pkg: the fixture)

pytestmark = pytest.mark.gpu


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(n, seed):
    return torch.randn(n, 512, generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()


@pytest.fixture(scope="module")
def blk(pkg):  # noqa: F811
    return make_block(pkg, heads=16)


def service(pkg, blk, lens=(40, 25, 33)):  # noqa: F811
    cache = pkg.LatentCache(n_pages=12, n_requests=len(lens), max_tokens=64, page_size=16)
    x = rows(sum(lens), 1)
    cu = [sum(lens[:b]) for b in range(len(lens) + 1)]
    step = cache.plan(i32(*lens), sum(lens))
    blk.prefill(x, cache.pages[0], step, cu)
    pkg.laga.check_status(step.status)
    return cache, [x[a:b] for a, b in zip(cu[:-1], cu[1:])]


@pytest.mark.parametrize("new,n,cu", [((10, 0, 0), 10, [0, 10]),              # request 0 holds tokens
                                      ((0, 3, 10), 13, [0, 3, 13]),           # one of two does not (it was released)
                                      ((0, 10, 0), 10, [0, 4, 10]),           # other lengths than the plan's
                                      ((0, 200, 0), 10, [0, 10])])            # a plan that could not be placed
def test_prefill_of_another_step_is_refused(pkg, blk, new, n, cu):  # noqa: F811
    laga = pkg.laga
    cache, _ = service(pkg, blk)
    cache.release(1)
    before = cache.pages[0].clone()
    step = cache.plan(i32(*new), max(n, 10))
    y = blk.prefill(rows(n, 2), cache.pages[0], step, cu)
    code, detail = laga.query_status(step.status)
    assert code == laga.ERR_CACHE_PLAN and detail == (0x50000003 if max(new) == 200 else 0x50000005)
    assert torch.equal(cache.pages[0], before) and bool(y.isnan().all())


@pytest.mark.parametrize("cu,pad", [([0, 10], 0), (None, 0), ([0, 10, 16], 6), ([0, 16], 6), ([0, 0, 10, 10], 0)])
def test_prefill_of_its_own_step_is_not(pkg, blk, cu, pad):  # noqa: F811
    """A released row again, padded or not, with boundaries given or one sequence."""
    cache, _ = service(pkg, blk)
    cache.release(1)
    step = cache.plan(i32(0, 10, 0), 10 + pad)
    x = rows(10 + pad, 3)
    y = blk.prefill(x, cache.pages[0], step, cu)
    pkg.laga.check_status(step.status)
    assert rel_l2(y[:10], blk(x[:10]).detach()) <= 1e-6


def test_prefill_in_two_calls(pkg, blk):  # noqa: F811
    """One plan of two prompts, run one prompt at a time: the first rows, then a plan whose rows begin behind them."""
    x = rows(50, 6)
    whole, halves = (pkg.LatentCache(n_pages=12, n_requests=2, max_tokens=64, page_size=16) for _ in range(2))
    step = whole.plan(i32(30, 20), 50)
    y = blk.prefill(x, whole.pages[0], step, [0, 30, 50])
    step = halves.plan(i32(30, 20), 50)
    a = blk.prefill(x[:30], halves.pages[0], step, [0, 30])
    b = blk.prefill(x[30:], halves.pages[0], step._replace(positions=step.positions[30:], slots=step.slots[30:]), [0, 20])
    pkg.laga.check_status(step.status)
    assert rel_l2(torch.cat([a, b]), y) <= 1e-6 and torch.equal(halves.pages[0], whole.pages[0])


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("new,right", [((1, 0, 1), [0]), ((0, 1, 1), []), ((2, 0, 1), [2]), ((1, 2, 0), [0]), ((1, 1, 1), [0, 1, 2])])
def test_decode_of_rows_that_are_not_their_requests(pkg, blk, new, right, plain):  # noqa: F811
    laga = pkg.laga
    cache, prompts = service(pkg, blk)
    before = cache.pages[0].clone()
    step = cache.plan(i32(*new), 3)
    laga.check_status(step.status)
    if plain:
        step = laga.CachePlan._make(step)
    token = rows(3, 4)
    ws = laga.alloc_workspace(laga.paged_decode_workspace_bytes(3, 16))
    y = blk.decode(token, cache.pages[0], step, cache.block_table, workspace=ws)
    changed = (cache.pages[0] != before).any(-1).view(-1).nonzero().view(-1).tolist()
    assert sorted(changed) == sorted(step.slots[b].item() for b in right)
    assert laga.query_status(ws)[0] == (laga.OK if len(right) == 3 else laga.ERR_DEVICE_CHECK)
    for b in range(3):
        if b in right:             # 2e-2: as in the service's test against one pass
            assert rel_l2(y[b], blk(torch.cat([prompts[b], token[b:b + 1]]))[-1].detach()) <= 2e-2
        else:
            assert not y[b].any()


def test_decode_after_a_plan_that_was_not_placed(pkg, blk):  # noqa: F811
    laga = pkg.laga
    cache, _ = service(pkg, blk)
    cache.n_free.zero_()
    before = cache.pages[0].clone()
    step = cache.plan(i32(30, 1, 1), 3)
    assert laga.query_status(step.status)[0] == laga.ERR_CACHE_PLAN
    ws = laga.alloc_workspace(laga.paged_decode_workspace_bytes(3, 16))
    y = blk.decode(rows(3, 5), cache.pages[0], step, cache.block_table, workspace=ws)
    assert laga.query_status(ws)[0] == laga.ERR_DEVICE_CHECK and not y.any() and torch.equal(cache.pages[0], before)
