"""The MLP branch of a Falcon decoder layer, trained with its activations saved
in 8 bits: z = x + W2 gelu(W1 norm(x)).

Algorithm 1's L_i.forward() and L_i.backward() for one rank whose layer has been
gathered: the weights are one flat bf16 vector (the layer that the gather
writes), their gradients one flat fp32 vector (what the partition step and the
qgZ quantizers take).  The plain products are torch's; everything around them is
`zpp`'s.

Between the passes the branch keeps, for every token, its input, the norm's
output and GELU's input as 8-bit checkpoints (1 + 1/64 bytes an element) and the
norm's two statistics.  GELU's output is computed again in its backward pass.
The first product's weight gradient comes straight from the checkpoint of the
norm's output, so both products' gradients are ready, and their exchange can
start, before the norm's backward pass.

    python -m paper_2407_01614_amd.mlp_layer --steps 20
"""
import argparse

import torch

from . import zpp


class MlpLayer:
    """Buffers and passes of one branch for batches of `tokens`."""

    def __init__(self, tokens, hidden, mlp, eps=1e-5, device="cuda"):
        self.tokens, self.hidden, self.mlp, self.eps = tokens, hidden, mlp, eps
        n = 2 * hidden + 2 * hidden * mlp
        self.weights = torch.empty(n, dtype=torch.bfloat16, device=device)
        self.grad = torch.zeros(n, dtype=torch.float32, device=device)
        self.gamma, self.beta, self.w1, self.w2 = self._split(self.weights)
        self.dgamma, self.dbeta, self.dw1, self.dw2 = self._split(self.grad)

        def matrix(cols):
            return torch.empty(tokens, cols, dtype=torch.bfloat16, device=device)

        def workspace(size):
            return torch.empty(size, dtype=torch.uint8, device=device)

        # kept between the passes
        self.x8 = zpp.empty_checkpoint(tokens, hidden, device)
        self.h8 = zpp.empty_checkpoint(tokens, hidden, device)
        self.u8 = zpp.empty_checkpoint(tokens, mlp, device)
        self.mean = torch.empty(tokens, dtype=torch.float32, device=device)
        self.rstd = torch.empty(tokens, dtype=torch.float32, device=device)
        # within a pass
        self.h = matrix(hidden)
        self.wide = [matrix(mlp) for _ in range(3)]
        self.norm_ws = workspace(zpp.layer_norm_backward_workspace(tokens, hidden))
        self.grad_ws = workspace(max(zpp.weight_grad_workspace(tokens, mlp, hidden),
                                     zpp.weight_grad_workspace(tokens, hidden, mlp)))

    def _split(self, flat):
        h, m = self.hidden, self.mlp
        gamma, beta, w1, w2 = flat.split([h, h, m * h, h * m])
        return gamma, beta, w1.view(m, h), w2.view(h, m)

    def saved_bytes(self):
        """Bytes kept between the passes."""
        kept = [*self.x8, *self.h8, *self.u8, self.mean, self.rstd]
        return sum(t.numel() * t.element_size() for t in kept)

    def forward(self, x, z):
        """z of x, both [tokens, hidden] bf16."""
        u, a, _ = self.wide
        zpp.layer_norm_forward(x, self.gamma, self.beta, self.h, self.mean, self.rstd,
                               eps=self.eps, saved=self.x8)
        zpp.checkpoint_save(self.h, self.h8)
        torch.mm(self.h, self.w1.t(), out=u)
        zpp.gelu_forward(u, a, saved=self.u8)
        torch.addmm(x, a, self.w2.t(), out=z)

    def backward(self, dz, dx, accumulate=False):
        """dx of dz; the weights' gradients into `grad`, or added to it."""
        da, du, a = self.wide
        torch.mm(dz, self.w2, out=da)
        zpp.gelu_backward(da, self.u8, du, a=a)
        zpp.weight_grad(dz, a, self.dw2, self.grad_ws, accumulate=accumulate)
        zpp.weight_grad(du, self.h8, self.dw1, self.grad_ws, accumulate=accumulate)
        torch.mm(du, self.w1, out=self.h)
        zpp.layer_norm_backward(self.h, self.x8, self.gamma, self.mean, self.rstd, dx,
                                self.dgamma, self.dbeta, self.norm_ws, dresidual=dz,
                                accumulate=accumulate)


def train(steps, tokens=512, hidden=256, mlp=1024, lr=2e-3, seed=0, log=None):
    """Fits the branch to another of the same shape on random tokens, with the
    framework's partition step as optimizer; the losses of the steps."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * std

    layer, goal = MlpLayer(tokens, hidden, mlp), MlpLayer(tokens, hidden, mlp)
    for net in (layer, goal):
        net.weights.copy_(normal(net.weights.numel(), std=hidden ** -0.5))
        net.gamma.fill_(1)
        net.beta.fill_(0)
    master = layer.weights.float()
    m, v = torch.zeros_like(master), torch.zeros_like(master)
    z, want, dx = (torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
                   for _ in range(3))
    losses = []
    for step in range(1, steps + 1):
        x = normal(tokens, hidden).to(torch.bfloat16)
        goal.forward(x, want)
        layer.forward(x, z)
        off = z.float() - want.float()
        losses.append(off.square().mean())
        layer.backward((off * (2.0 / off.numel())).to(torch.bfloat16), dx)
        zpp.adam_partition_step(master, m, v, layer.grad, layer.weights, lr=lr, beta1=0.9,
                                beta2=0.95, eps=1e-10, weight_decay=0.0, step=step)
        if log:
            log("step %d: loss %.5f" % (step, float(losses[-1])))
    return [float(x) for x in losses]


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--hidden", type=int, default=256)
    p.add_argument("--mlp", type=int, default=1024)
    args = p.parse_args()
    train(args.steps, args.tokens, args.hidden, args.mlp, log=print)


if __name__ == "__main__":
    main()
