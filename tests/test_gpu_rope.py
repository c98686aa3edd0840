"""Rotary positions and the latent-norm-with-rotation step on the GPU against float64 references."""
import pytest
import torch

import serving_reference as ref
from parity import f64

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def laga():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_17644_b200 import laga as _laga
    _laga.lib()
    return _laga


def within(got, want, bound, what=""):
    err = (f64(got) - want).abs()
    assert not torch.isnan(f64(got)).any(), what
    over = err - bound
    assert float(over.max()) <= 0, f"{what}: error {float(err.flatten()[over.argmax()]):.3e} over its bound {float(bound.flatten()[over.argmax()]):.3e}"


def plan_of(laga, d_rot, interleaved, scaled=False):
    return laga.rope_plan(d_rot, scaling={"type": "yarn", "factor": 40} if scaled else None, interleaved=interleaved)


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("M,h,d,begin,d_rot", [(1, 1, 64, 0, 64), (1, 16, 192, 128, 64), (7, 3, 192, 128, 64), (513, 16, 192, 128, 64),
                                               (40, 1, 64, 0, 64), (1000, 1, 64, 0, 64), (5, 128, 192, 128, 64), (33, 5, 128, 32, 32),
                                               (2100, 1, 16, 0, 16), (9, 2, 1024, 8, 256), (300, 7, 96, 0, 96), (3, 1000, 24, 8, 16)])
def test_rope(laga, interleaved, M, h, d, begin, d_rot):
    g = torch.Generator().manual_seed(M * 131 + h)
    x = torch.randn(M, h, d, generator=g).to(BF16)
    pos = torch.randint(-5, 5_000_000, (M,), generator=g, dtype=torch.int32)
    rope = plan_of(laga, d_rot, interleaved, scaled=M % 2 == 1)
    fr = rope.freqs.cpu()
    for inverse in (False, True):
        want, bound = ref.rotate(x.double(), pos, fr, rope.mscale, interleaved, inverse, begin)
        y = torch.full((M, h, d), float("nan"), dtype=BF16, device="cuda")
        laga.rope(x.cuda(), pos.cuda(), rope, rot_begin=begin, inverse=inverse, y=y)
        within(y, want, bound)
        z = x.cuda()
        assert laga.rope(z, pos.cuda(), rope, rot_begin=begin, inverse=inverse, y=z) is z
        assert torch.equal(z, y)                                     # in place: the same bits


@pytest.mark.parametrize("interleaved", [True, False])
def test_rope_strided_rows_and_neighbours(laga, interleaved):
    """The shared key where W_kv_a leaves it (a column slice), in place and out of place, and rows of a wider output:
    what lies between the rows stays."""
    M = 77
    kv = torch.randn(M, 576, generator=torch.Generator().manual_seed(1)).to(BF16)
    pos = torch.arange(M, dtype=torch.int32)
    rope = plan_of(laga, 64, interleaved)
    want, bound = ref.rotate(kv[:, None, 512:].double(), pos, rope.freqs.cpu(), 1.0, interleaved)
    dev = kv.cuda()
    view = dev[:, 512:].unsqueeze(1)
    y = laga.rope(view, pos.cuda(), rope)
    within(y, want, bound)
    wide = torch.full((M, 3, 64), 7.0, dtype=BF16, device="cuda")
    laga.rope(view, pos.cuda(), rope, y=wide[:, 1:2])
    assert torch.equal(wide[:, 1:2], y) and bool((wide[:, 0] == 7).all() and (wide[:, 2] == 7).all())
    laga.rope(view, pos.cuda(), rope, y=view)
    assert torch.equal(view, y) and torch.equal(dev[:, :512].cpu(), kv[:, :512])
    with pytest.raises(laga.LagaError):                              # overlapping, not the same
        laga.rope(dev[:, 448:512].unsqueeze(1), pos.cuda(), rope, y=dev[:, 512:].unsqueeze(1))
    with pytest.raises(ValueError):                                  # heads that are not dense
        laga.rope(torch.zeros(4, 8, 128, dtype=BF16, device="cuda")[:, ::2], pos[:4].cuda(), rope)
    with pytest.raises(ValueError):
        laga.rope(y, pos.cuda().long(), rope)


def test_rope_gradient_is_the_transpose(laga):
    """<R x, dy> = <x, R^T dy>, and differences: R is linear, so R(x + e) - R(x) = R e, whose product with dy the inverse call
    gives.  Products are formed in float64 from bf16 outputs: each output is off by U relative, so the sums by U times the
    sums of magnitudes."""
    M, h = 50, 4
    g = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(M, h, 192, generator=g).to(BF16) for _ in range(2))
    pos = torch.randint(0, 100_000, (M,), generator=g, dtype=torch.int32).cuda()
    for interleaved in (True, False):
        rope = plan_of(laga, 64, interleaved, scaled=True)
        a = f64(laga.rope(x.cuda(), pos, rope)) * dy.double()
        b = f64(laga.rope(dy.cuda(), pos, rope, inverse=True)) * x.double()
        assert abs(float(a.sum() - b.sum())) <= 1.01 * ref.U * float(a.abs().sum() + b.abs().sum())


def latent_case(M, D, R, seed, with_beta):
    g = torch.Generator().manual_seed(seed)
    kv = torch.randn(M, D + R, generator=g) * (0.5 + 2 * torch.rand(M, 1, generator=g)) + torch.randn(M, 1, generator=g)
    gamma = (1 + 0.2 * torch.randn(D, generator=g)).to(BF16)
    beta = (0.1 * torch.randn(D, generator=g)).to(BF16) if with_beta else None
    pos = torch.randint(0, 200_000, (M,), generator=g, dtype=torch.int32)
    return kv.to(BF16), gamma, beta, pos, torch.randn(M, D, generator=g).to(BF16), torch.randn(M, R, generator=g).to(BF16)


SHAPES = [(1, 512, 64, True), (2, 512, 64, False), (777, 512, 64, True), (5000, 512, 64, True), (65, 8, 16, True), (100, 264, 128, False),
          (300, 1024, 256, True), (33, 256, 32, False)]


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("M,D,R,with_beta", SHAPES)
def test_latent_norm_rope_forward_and_backward(laga, interleaved, M, D, R, with_beta):
    kv, gamma, beta, pos, dl, dk = latent_case(M, D, R, M + D, with_beta)
    rope = plan_of(laga, R, interleaved, scaled=M % 2 == 0)
    dev = [t.cuda() if t is not None else None for t in (kv, gamma, beta, pos)]
    nan = lambda *s: torch.full(s, float("nan"), dtype=BF16, device="cuda")  # noqa: E731
    latent, k_pe, mean, rstd = laga.latent_norm_rope(*dev, rope, latent=nan(M, D), k_pe=nan(M, R))
    y, rmean, rrstd, bound = ref.norm(kv[:, :D].double(), gamma.double(), None if beta is None else beta.double(), 1e-5)
    within(latent, y, bound, "latent")
    spread = kv[:, :D].double().abs().mean(1)
    within(mean, rmean, D * 2.0 ** -24 * spread, "mean")
    within(rstd, rrstd, D * 2.0 ** -22 * rrstd * (1 + spread * rrstd), "rstd")
    fr = rope.freqs.cpu()
    within(k_pe, *ref.rotate(kv[:, D:].double(), pos, fr, rope.mscale, interleaved), "k_pe")

    args = (dl.cuda(), dk.cuda(), dev[0], dev[1], mean, rstd, dev[3], rope)
    dkv, dgamma, dbeta = laga.latent_norm_rope_backward(*args, with_beta=with_beta, dkv_a=nan(M, D + R))
    dx, rg, rb, bound, mag_g, mag_b = ref.norm_backward(dl.double(), kv[:, :D].double(), gamma.double(), f64(mean), f64(rstd))
    within(dkv[:, :D], dx, bound, "dx")
    within(dkv[:, D:], *ref.rotate(dk.double(), pos, fr, rope.mscale, interleaved, inverse=True), "dk")
    # sums: a chain of M / 2368 rows, 8 warps, 37 blocks, 8 warps, each addition off by 2^-24 of sums below the magnitudes'
    chain = (M / 2368 + 64) * 2.0 ** -24
    within(dgamma, rg, chain * mag_g + 2.0 ** -22 * mag_g + 1e-30, "dgamma")
    if with_beta:
        within(dbeta, rb, chain * mag_b + 1e-30, "dbeta")
    else:
        assert dbeta is None
    again = laga.latent_norm_rope_backward(*args, with_beta=with_beta)
    assert torch.equal(again[0], dkv) and torch.equal(again[1], dgamma)                # bit for bit


def test_latent_norm_rope_gradients_by_differences(laga):
    """Central differences of <latent, dl> + <k_pe, dk> in float64 (the reference forward) against the kernel's gradient:
    the reference's own derivative is the formula's, checked here independently of it."""
    M, D, R = 3, 16, 16
    kv, gamma, beta, pos, dl, dk = latent_case(M, D, R, 5, True)
    rope = plan_of(laga, R, True)
    _, _, mean, rstd = laga.latent_norm_rope(kv.cuda(), gamma.cuda(), beta.cuda(), pos.cuda(), rope)
    dkv, dgamma, dbeta = laga.latent_norm_rope_backward(dl.cuda(), dk.cuda(), kv.cuda(), gamma.cuda(), mean, rstd, pos.cuda(), rope)

    def value(kv_, gamma_, beta_):
        y = ref.norm(kv_[:, :D], gamma_, beta_, 1e-5)[0]
        k = ref.rotate(kv_[:, D:], pos, rope.freqs.cpu(), 1.0, True)[0]
        return float((y * dl.double()).sum() + (k * dk.double()).sum())

    base = [kv.double(), gamma.double(), beta.double()]
    for which, grad in ((0, dkv), (1, dgamma), (2, dbeta)):
        flat = f64(grad).flatten()
        for i in range(flat.numel()):
            moved = []
            for step in (1e-5, -1e-5):
                t = [b.clone() for b in base]
                t[which].view(-1)[i] += step
                moved.append(value(*t))
            numeric = (moved[0] - moved[1]) / 2e-5
            # U for the rounding to bf16, 1e-4 for fp32 arithmetic and the quotient (values of order ten: 1e-15 * 10 / 1e-5)
            assert abs(float(flat[i]) - numeric) <= ref.U * abs(numeric) + 1e-4


def test_strided_input_and_cache_rows(laga):
    """kv_a inside a wider matrix; rows into the cache and dense at once, and into the cache alone; padding slots, rows
    no slot names, and slots outside the cache leave it untouched."""
    M, D, R = 70, 512, 64
    kv, gamma, beta, pos, _, _ = latent_case(M, D, R, 9, True)
    wide = torch.full((M, 640), float("nan"), dtype=BF16, device="cuda")
    wide[:, :576] = kv.cuda()
    rope = plan_of(laga, 64, True)
    slots = torch.randperm(10 * 16, generator=torch.Generator().manual_seed(2))[:M].to(torch.int32)
    slots[5], slots[6], slots[-1] = -1, 160, -2147483648
    start = torch.full((10, 16, 576), 3.0, dtype=BF16, device="cuda")
    args = (wide[:, :576], gamma.cuda(), beta.cuda(), pos.cuda(), rope)
    both = start.clone()
    latent, k_pe, mean, rstd = laga.latent_norm_rope(*args, cache=both, slots=slots.cuda())
    dense = laga.latent_norm_rope(kv.cuda(), *args[1:])
    for a, b in zip((latent, k_pe, mean, rstd), dense):
        assert torch.equal(a, b)
    want = start.cpu().view(-1, 576)
    ok = (slots >= 0) & (slots < 160)
    want[slots[ok].long()] = torch.cat([latent, k_pe], 1).cpu()[ok]
    assert torch.equal(both.cpu().view(-1, 576), want)
    alone = start.clone()
    assert laga.cache_append(*args, slots.cuda(), alone) is alone and torch.equal(alone, both)
    with pytest.raises(ValueError):
        laga.cache_append(*args, slots.cuda().long(), alone)
    with pytest.raises(ValueError):
        laga.cache_append(*args, slots.cuda(), alone[..., :512])


def test_empty_batches(laga):
    rope = plan_of(laga, 64, True)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert laga.rope(torch.zeros(0, 4, 192, dtype=BF16, device="cuda"), none, rope).shape == (0, 4, 192)
    kv, gamma = torch.zeros(0, 576, dtype=BF16, device="cuda"), torch.ones(512, dtype=BF16, device="cuda")
    latent, k_pe, mean, rstd = laga.latent_norm_rope(kv, gamma, None, none, rope)
    assert latent.shape == (0, 512) and k_pe.shape == (0, 64)
    dkv, dgamma, dbeta = laga.latent_norm_rope_backward(latent, k_pe, kv, gamma, mean, rstd, none, rope)
    assert dkv.shape == (0, 576) and not dgamma.any() and not dbeta.any()


def test_given_buffers_come_back_and_plans_are_checked(laga):
    plan = laga.rope_plan(64)
    x, pos = torch.randn(5, 2, 192, device="cuda").to(BF16), torch.arange(5, dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    assert laga.rope(x, pos, plan, y=y) is y and torch.equal(laga.rope(x, pos, plan), y)
    assert laga.rope(x, pos, plan, y=x) is x and torch.equal(x, y)
    for wrong in ((plan.freqs, 1.0), plan.freqs, None):
        with pytest.raises(TypeError):
            laga.rope(x, pos, wrong)
    for freqs in (plan.freqs.float(), plan.freqs.cpu(), plan.freqs.repeat(2)[::2]):
        with pytest.raises(ValueError):
            laga.rope(x, pos, laga.RopePlan(freqs))
    for positions in (pos.long(), pos[:4], pos.cpu()):
        with pytest.raises(ValueError):
            laga.rope(x, positions, plan)
    with pytest.raises(ValueError):
        laga.rope(x, pos, plan, y=y[:4])
    with pytest.raises(laga.LagaError):
        laga.rope(x, pos, plan, rot_begin=136)
    kv, gamma = torch.randn(5, 576, device="cuda").to(BF16), torch.ones(512, dtype=BF16, device="cuda")
    latent, k_pe = torch.empty(5, 512, dtype=BF16, device="cuda"), torch.empty(5, 64, dtype=BF16, device="cuda")
    out = laga.latent_norm_rope(kv, gamma, None, pos, plan, latent=latent, k_pe=k_pe)
    assert out[0] is latent and out[1] is k_pe and out[2].shape == out[3].shape == (5,)
    with pytest.raises(laga.LagaError):                              # an output over another
        laga.latent_norm_rope(kv, gamma, None, pos, plan, latent=latent, k_pe=latent.view(-1)[:320].view(5, 64))
    with pytest.raises(ValueError):
        laga.latent_norm_rope(kv, gamma[:504], None, pos, plan)
