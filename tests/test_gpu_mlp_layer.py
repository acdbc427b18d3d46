"""The MLP branch on 8-bit checkpoints (paper_2407_01614_amd.mlp_layer) as one
path: its gradients against float64 autograd of the same branch, gradients added
up over two batches, and a short training run."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mlp_layer():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_01614_amd import mlp_layer as mod
    return mod


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


# How far off the gradients may be, as a share of their norms.  bf16 keeps 2^-9 of
# a number on average over five roundings in a row: below 1%.  A checkpoint's step
# is at most 2 / 127 of a block's largest magnitude, 2.5 to 3 standard deviations of
# 64 normal numbers, so its error is 0.04 / sqrt(12) = 1.2% of one; two of them
# (GELU's input with its output, the norm's) meet in a gradient.
BOUND = 0.03


@pytest.mark.parametrize("tokens,hidden,mlp", [(96, 64, 256), (257, 200, 520)])
def test_gradients(mlp_layer, tokens, hidden, mlp):
    gen = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    layer = mlp_layer.MlpLayer(tokens, hidden, mlp)
    layer.weights.copy_(normal(layer.weights.numel()) * hidden ** -0.5)
    layer.gamma.copy_(1 + 0.1 * normal(hidden))
    x, dz = normal(tokens, hidden).to(torch.bfloat16), normal(tokens, hidden).to(torch.bfloat16)
    z, dx = torch.empty_like(x), torch.empty_like(x)
    layer.forward(x, z)
    layer.backward(dz, dx)

    p = [t.double().requires_grad_() for t in (x, layer.gamma, layer.beta, layer.w1, layer.w2)]
    xd, g, b, w1, w2 = p
    mean = xd.mean(1, keepdim=True)
    h = (xd - mean) / torch.sqrt((xd - mean).square().mean(1, keepdim=True) + layer.eps) * g + b
    u = h @ w1.t()
    out = xd + (u * 0.5 * torch.special.erfc(-u * 0.5 ** 0.5)) @ w2.t()
    out.backward(dz.double())
    assert rel(z, out.detach()) < 0.01
    for name, got, want in zip(("dx", "dgamma", "dbeta", "dw1", "dw2"),
                               (dx, layer.dgamma, layer.dbeta, layer.dw1, layer.dw2), p):
        assert rel(got, want.grad) < BOUND, name
    # another batch's added: twice the same here
    once = layer.grad.clone()
    layer.backward(dz, dx, accumulate=True)
    assert torch.equal(layer.grad, 2 * once)
    # half of what bf16 would keep
    assert layer.saved_bytes() < 0.55 * 2 * tokens * (2 * hidden + mlp) + 8 * tokens


def test_training(mlp_layer):
    losses = mlp_layer.train(30)
    assert losses[-1] < 0.5 * losses[0] and all(l == l for l in losses)
