"""What the kernels of a service report reaches the caller of the block."""
import pytest
import torch

from test_gpu_serving import BF16, make_block, pkg  # noqa: F401  (pkg: the fixture)

pytestmark = pytest.mark.gpu


def test_status_of_prefill_and_decode(pkg):  # noqa: F811
    """The attention's status of both, clean and with a table entry that names no page (which reads as zeros)."""
    laga = pkg.laga
    blk = make_block(pkg, heads=16)
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.randn(62, 512, generator=torch.Generator().manual_seed(8)).to(BF16).cuda()
    cache = pkg.LatentCache(n_pages=6, n_requests=2, max_tokens=64, page_size=16)
    ws = laga.alloc_workspace(laga.fwd_varlen_workspace_bytes(60, 2, 16))
    ws[:4] = 0xff
    step = cache.plan(torch.tensor([40, 20], **i32), 60)
    y = blk.prefill(x[:60], cache.pages[0], step, [0, 40, 60], workspace=ws)
    laga.check_status(step.status)
    laga.check_status(ws)
    again = blk.prefill(x[:60], cache.pages[0], step, [0, 40, 60])
    assert torch.equal(y, again)
    ws = laga.alloc_workspace(laga.paged_decode_workspace_bytes(2, 16))
    step = cache.plan(torch.ones(2, **i32), 2)
    good = blk.decode(x[60:], cache.pages[0], step, cache.block_table, workspace=ws)
    laga.check_status(ws)
    cache.block_table[0, 1] = 6
    bad = blk.decode(x[60:], cache.pages[0], step, cache.block_table, workspace=ws)
    with pytest.raises(laga.LagaError) as err:
        laga.check_status(ws)
    assert err.value.code == laga.ERR_DEVICE_CHECK and torch.equal(bad[1], good[1])
