"""Second derivatives, which the library does not have, raise; first derivatives under create_graph are the ordinary ones."""
import pytest
import torch

from test_gpu_serving import BF16, pkg  # noqa: F401  (pkg: the fixture)

pytestmark = pytest.mark.gpu


def functions(pkg):  # noqa: F811
    from paper_2607_17644_b200 import block
    g = torch.Generator().manual_seed(4)

    def t(*shape):
        return (torch.randn(*shape, generator=g) * 0.5).to(BF16).cuda().requires_grad_(True)

    pos, rope = torch.arange(40, dtype=torch.int32, device="cuda"), pkg.laga.rope_plan(64)
    return {"rotary": (lambda x: block.rotary(x, pos, rope), [t(40, 2, 192)]),
            "latent_norm_rope": (lambda kv, a, b: torch.cat(block.latent_norm_rope(kv, a, b, pos, rope), 1), [t(40, 576), t(512), t(512)]),
            "linear": (block.linear, [t(40, 64), t(64, 128)]),
            "layernorm": (block.layernorm, [t(40, 512), t(512), t(512)]),
            "attention": (pkg.laga_attention, [t(40, 2, 192), t(40, 512), t(40, 64), t(512, 512)])}


@pytest.mark.parametrize("name", ["rotary", "latent_norm_rope", "linear", "layernorm", "attention"])
def test_second_derivatives_raise(pkg, name):  # noqa: F811
    f, inputs = functions(pkg)[name]
    loss = f(*inputs).float().square().sum()
    first = torch.autograd.grad(loss, inputs, retain_graph=True)
    again = torch.autograd.grad(loss, inputs, create_graph=True)
    for a, b in zip(first, again):
        # (weight gradients of the attention and of a linear may add in another order: 2^-8 is bf16's half step)
        assert float((a - b).detach().float().norm()) <= 2.0 ** -8 * float(a.float().norm()) and b.requires_grad
    with pytest.raises(RuntimeError, match="second derivatives"):
        sum(b.float().square().sum() for b in again).backward()


@pytest.mark.parametrize("name", ["latent_norm_rope", "layernorm", "attention"])
def test_also_where_only_what_was_saved_is_differentiated(pkg, name):  # noqa: F811
    """A loss linear in the output: the incoming gradient is a constant, the gradient still depends on the inputs."""
    f, inputs = functions(pkg)[name]
    grads = torch.autograd.grad(f(*inputs).float().sum(), inputs, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (grads[0].float().square().sum() + inputs[0].float().sum()).backward()
