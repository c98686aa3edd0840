"""The block's softmax scale: the same in training, prefill and decode, and with it YaRN's factor on whole scores."""
import math

import pytest
import torch

import serving_reference as ref
from parity import rel_l2
from test_gpu_serving import BF16, bf, pkg  # noqa: F401  (pkg: the fixture)

pytestmark = pytest.mark.gpu


def make(pkg, factor, heads=4):  # noqa: F811
    rope = pkg.laga.rope_plan(64, scaling={"type": "yarn", "factor": factor, "mscale_weight": 0})
    scale = 192 ** -0.5 * (0.1 * math.log(factor) + 1) ** 2
    return pkg.LagaBlock(512, heads, seed=5, rope=rope, softmax_scale=scale), scale


def test_training_with_a_scale_of_the_callers(pkg, oracle):  # noqa: F811
    """As the block's test with rotation, with the scale given; tolerances are that test's."""
    blk, scale = make(pkg, 40)
    assert blk.rope.mscale == 1.0 and scale > 1.8 * 192 ** -0.5
    S, H = 200, blk.n_heads
    g = torch.Generator().manual_seed(17)
    hidden, d_out = (torch.randn(S, 512, generator=g).to(BF16) for _ in range(2))
    y = blk(hidden.cuda())
    y.backward(d_out.cuda())
    w_q, w_kv_a, w_kv_b, w_o = (p.detach().cpu() for p in (blk.w_q, blk.w_kv_a, blk.w_kv_b, blk.w_o))
    pos, freqs = torch.arange(S, dtype=torch.int32), blk.rope.freqs.cpu()
    turn = lambda t, inv=False: ref.rotate(t.double(), pos, freqs, 1.0, True, inv)[0]  # noqa: E731
    q = bf(turn(bf(oracle.linear(hidden, w_q)).view(S, H, 192)))
    kv_a = bf(oracle.linear(hidden, w_kv_a))
    latent = bf(oracle.layernorm(kv_a[:, :512].contiguous(), blk.ln_gamma.detach().cpu(), blk.ln_beta.detach().cpu(), blk.eps)[0])
    k_pe = bf(turn(kv_a[:, 512:]))
    out = oracle.fwd(q, latent, k_pe, w_kv_b, 128, scale, causal=True, kv_round_bf16=True)[0]
    out_b = bf(out).reshape(S, H * 128)
    assert rel_l2(y.detach(), oracle.linear(out_b, w_o)) <= 1e-2
    r = oracle.bwd(q, latent, k_pe, w_kv_b, bf(oracle.linear_bwd(d_out, out_b, w_o)[0]).view(S, H, 128), 128, scale, causal=True, kv_round_bf16=True)
    assert rel_l2(blk.w_kv_b.grad, r["dw"]) <= 2e-2
    assert rel_l2(blk.w_q.grad, oracle.linear_bwd(bf(turn(bf(r["dq"]), True)).reshape(S, H * 192), hidden, w_q)[1]) <= 2e-2


def test_service_with_a_scale_of_the_callers(pkg):  # noqa: F811
    """A prompt of 50 tokens and ten decode steps against the block's forward (2e-2: as in the service's own test against one pass)."""
    blk, _ = make(pkg, 16, heads=16)
    x = torch.randn(60, 512, generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    cache = pkg.LatentCache(n_pages=4, n_requests=1, max_tokens=64, page_size=16)
    prompt = blk.prefill(x[:50], cache.pages[0], cache.plan(torch.tensor([50], dtype=torch.int32, device="cuda"), 50), [0, 50])
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    rows = [blk.decode(x[i:i + 1], cache.pages[0], cache.plan(one, 1), cache.block_table) for i in range(50, 60)]
    whole = blk(x).detach()
    assert rel_l2(prompt, whole[:50]) <= 1e-6 and rel_l2(torch.cat(rows), whole[50:]) <= 2e-2
