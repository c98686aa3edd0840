"""No requests at all: the cache's plan and the one-token attention return empty results, as the rotary calls do."""
import pytest
import torch

from test_gpu_decode import BF16, laga  # noqa: F401  (laga: the fixture)

pytestmark = pytest.mark.gpu


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


def test_plan_of_no_requests(laga):  # noqa: F811
    free, n_free = torch.arange(5, dtype=torch.int32, device="cuda"), i32(1) + 4
    p = laga.cache_plan(i32(0), i32(0), i32(0, 3), free, n_free, 16, 7)
    laga.check_status(p.status)
    assert p.slots.tolist() == [-1] * 7 and p.positions.tolist() == [0] * 7 and p.cu_new_lens.tolist() == [0]
    assert p.seq_lens.shape == (0,) and p.n_free.tolist() == [4] and n_free.tolist() == [4] and free.tolist() == list(range(5))
    for t in p:
        t.fill_(77)
    q = laga.cache_plan(i32(0), i32(0), i32(0, 3), free, n_free, 16, 7, out=p)
    assert q is p and p.slots.tolist() == [-1] * 7 and p.positions.tolist() == [0] * 7 and p.cu_new_lens.tolist() == [0]
    assert p.n_free.tolist() == [4] and p.status.tolist() == [0]
    with pytest.raises(laga.LagaError):
        laga.cache_plan(i32(0), i32(0), i32(0, 3), free, n_free, 24, 7)
    with pytest.raises(ValueError):
        laga.cache_plan(i32(0), i32(1), i32(0, 3), free, n_free, 16, 7)


def test_decode_of_no_requests(laga):  # noqa: F811
    q, w = torch.zeros(0, 16, 192, dtype=BF16, device="cuda"), torch.zeros(512, 4096, dtype=BF16, device="cuda")
    cache = torch.zeros(2, 16, 576, dtype=BF16, device="cuda")
    lse, out = torch.zeros(0, 16, device="cuda"), torch.zeros(0, 16, 128, dtype=BF16, device="cuda")
    for given in (None, laga.alloc_workspace(laga.paged_decode_workspace_bytes(1, 16)).fill_(0xff)):
        got, got_lse, ws = laga.paged_decode(q, w, cache, i32(0, 3), i32(0), lse=lse, workspace=given)
        laga.check_status(ws)
        assert got.shape == (0, 16, 128) and got.dtype == BF16 and got_lse is lse and (given is None or ws is given)
    assert laga.paged_decode(q, w, cache, i32(0, 3), i32(0), out=out)[0] is out
    with pytest.raises(laga.LagaError) as err:                       # another geometry, and no requests of it
        laga.paged_decode(q[..., :64], w[:, :16 * 64].contiguous(), cache, i32(0, 3), i32(0))
    assert err.value.code == laga.ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        laga.paged_decode(q, w, cache, i32(1, 3), i32(0))
