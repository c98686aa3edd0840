"""The rotary, cache and decode calls from several threads at once, a training step of the rotary block in a graph, and the decode kernel's
time through the profiling slots."""
import threading

import pytest
import torch

from test_gpu_decode import case, laga  # noqa: F401  (laga: the fixture)
from test_gpu_serving import BF16, make_block, pkg  # noqa: F401  (pkg: the fixture)

pytestmark = pytest.mark.gpu


def test_calls_from_two_threads(laga):  # noqa: F811
    """Each thread on a stream of its own with tensors of its own, the binding letting the other run meanwhile: the results of the calls alone."""
    def work(seed, lens, h, rounds):
        q, w, cache, table, n = (t.cuda() for t in case(lens, h, 16, seed=seed, fill=0.0))
        rope, B = laga.rope_plan(64), len(lens)
        pos, slots = n - 1, torch.arange(B, dtype=torch.int32, device="cuda")
        kv = torch.randn(B, 576, generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()
        gamma, free = torch.ones(512, dtype=BF16, device="cuda"), torch.arange(64, dtype=torch.int32, device="cuda")
        held = torch.zeros(B, 8, dtype=torch.int32, device="cuda")
        out = []
        for _ in range(rounds):
            x = laga.rope(q, pos, rope)
            pages = laga.cache_append(kv, gamma, None, pos, rope, slots, cache.clone())
            plan = laga.cache_plan(torch.zeros_like(n), torch.ones_like(n), held.clone(), free, torch.full_like(n[:1], 64), 16, B)
            y, _, ws = laga.paged_decode(x, w, pages, table, n)
            latent, k_pe, mean, rstd = laga.latent_norm_rope(kv, gamma, None, pos, rope)
            grads = laga.latent_norm_rope_backward(latent, k_pe, kv, gamma, mean, rstd, pos, rope, with_beta=False)
            out.append((x, pages, plan.slots, plan.n_free, y, ws[:4].clone(), latent, k_pe, *grads[:2]))
        return out

    jobs = [(61, [300, 0, 17, 900], 16, 40), (62, [64, 65], 40, 40)]
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


@pytest.mark.parametrize("with_rope", [True, False])
def test_training_step_in_a_graph(pkg, with_rope):  # noqa: F811
    """forward and backward with positions given, captured and replayed on new inputs: the eager step's output and gradients (weights' gradients
    up to the order in which the GEMMs and the shared key's sums add: bf16's half step)."""
    blk = make_block(pkg, heads=2) if with_rope else pkg.LagaBlock(512, 2)
    S = 200
    pos = torch.arange(S, dtype=torch.int32, device="cuda") if with_rope else None
    g = torch.Generator().manual_seed(9)
    data = [[torch.randn(S, 512, generator=g).to(BF16).cuda() for _ in range(2)] for _ in range(3)]
    x, dy = (torch.zeros_like(t) for t in data[0])
    params = list(blk.parameters())

    def step():
        h = x.detach().requires_grad_(True)
        y = blk(h, positions=pos)
        return (y.detach(), *torch.autograd.grad(y, [h, *params], dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for a, b in data:
        x.copy_(a)
        dy.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        assert torch.equal(captured[0], eager[0])
        for got, want in zip(captured[1:], eager[1:]):
            assert float((got.float() - want.float()).norm()) <= 2.0 ** -8 * float(want.float().norm())


def test_decode_kernels_time_through_the_profiling_slots(laga):  # noqa: F811
    q, w, cache, table, n = (t.cuda() for t in case([3000, 700], 16, 64, seed=63, fill=0.0))
    events = [[torch.cuda.Event(enable_timing=True) for _ in range(2)] for _ in range(2)]
    for pair in events:
        for e in pair:
            e.record()
    laga.profile_kernel("attn_decode", events[0], events[1])
    try:
        for _ in range(2):
            ws = laga.paged_decode(q, w, cache, table, n)[2]
        laga.check_status(ws)
        torch.cuda.synchronize()
    finally:
        laga.profile_kernel("attn_decode")
    assert all(a.elapsed_time(b) > 0 for a, b in zip(*events))
