"""Plain 64-bit forms of the layer operators and the bounds that the kernels'
32-bit results have to keep, for tests/test_gpu_layers.py.

U is the unit roundoff of fp32.  A result rounded to bf16 adds half a bf16 ulp,
2^-8 of it at most.
"""
import numpy as np
import torch

U = 2.0 ** -24
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
# the smallest normal float: results below may be flushed
TINY = 2.0 ** -126
BLOCK = 64


def matrix(rows, cols, dtype, pad=0, offset=0, fill=None, device="cuda"):
    """A [rows, cols] view of a buffer `pad` features wider whose first element
    is `offset` elements into its allocation."""
    buf = torch.empty(rows * (cols + pad) + offset, dtype=dtype, device=device)
    if fill is not None:
        buf.fill_(fill)
    return buf[offset:].view(rows, cols + pad)[:, :cols]


def values(rows, cols, seed, dtype, pad=0, offset=0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    m = matrix(rows, cols, dtype, pad, offset)
    m.copy_(torch.randn(rows, cols, device="cuda", generator=gen) * std)
    return m


# --------------------------------------------------------------------------
# Checkpoints, in integers
# --------------------------------------------------------------------------
def encode(x):
    """Codes and exponents of a float32 numpy matrix, decided in exact integer
    and 64-bit arithmetic."""
    rows, cols = x.shape
    codes = np.zeros((rows, cols), np.int8)
    exps = np.zeros((rows, -(-cols // BLOCK)), np.uint8)
    for b in range(exps.shape[1]):
        part = x[:, b * BLOCK:(b + 1) * BLOCK].astype(np.float64)
        finite = np.isfinite(part).all(axis=1)
        top = np.where(finite, np.abs(np.where(np.isfinite(part), part, 0)).max(axis=1), 0.0)
        e = np.full(rows, -126)
        for k in range(-126, 122):   # the smallest e with top <= 127 * 2^e
            e = np.where(top > 127.0 * 2.0 ** k, k + 1, e)
        most = np.where(e >= 122, 63, 127)[:, None]
        c = np.rint(np.where(finite[:, None], part, 0.0) / (2.0 ** e.astype(np.float64))[:, None])
        codes[:, b * BLOCK:(b + 1) * BLOCK] = np.clip(c, -most, most)
        exps[:, b] = np.where(finite, e + 127, 255)
    return codes, exps


def decode(codes, exps):
    """The values of a checkpoint in float64 (numpy)."""
    scale = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    return codes.astype(np.float64) * np.repeat(scale, BLOCK, axis=1)[:, :codes.shape[1]]


def saved(x):
    """The checkpoint of a matrix as GPU tensors, and its values in float64."""
    codes, exps = encode(x.float().cpu().numpy())
    v = torch.from_numpy(decode(codes, exps)).cuda()
    return (torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda()), v


# --------------------------------------------------------------------------
# Layer norm
# --------------------------------------------------------------------------
def chain(cols):
    """Roundings that a sum over a row passes through, at most: a lane's own
    elements one after the other, then the lanes pairwise and by waves."""
    return 32 + cols / 1024 + 24


def norm_forward(s, gamma, beta, eps, dtype):
    """y, mean, rstd of float64 s, and the bounds of their errors."""
    cols = s.shape[1]
    mean = s.mean(1, keepdim=True)
    var = (s - mean).square().mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    y = (s - mean) * rstd * gamma + beta
    dmean = chain(cols) * U * s.abs().mean(1, keepdim=True)
    # the squares' sum, and what a mean off by dmean adds to it
    drel = 0.5 * ((chain(cols) + 4) * U + (dmean * rstd).square()) + 4 * U
    dy = (gamma * rstd).abs() * (dmean + (s - mean).abs() * (drel + 4 * U))
    dy = dy + 4 * U * (y.abs() + beta.abs()) + ROUND[dtype] * y.abs() * (1 + ROUND[dtype]) + TINY
    return (y, mean[:, 0], rstd[:, 0]), (dy, dmean[:, 0] + U * mean[:, 0].abs(),
                                         rstd[:, 0] * drel[:, 0])


def norm_backward(dy, x, gamma, beta, mean, rstd, dresidual, dtype):
    """dx, dgamma, dbeta, y in float64, and the bounds of their errors."""
    rows, cols = dy.shape
    mean, rstd = mean[:, None], rstd[:, None]
    h = (x - mean) * rstd
    g = dy * gamma
    c1, c2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = rstd * (g - c1 - h * c2)
    n = chain(cols) + 8
    err = rstd * (n * U * g.abs().mean(1, keepdim=True)
                  + h.abs() * n * U * (g * h).abs().mean(1, keepdim=True)
                  + 8 * U * (g.abs() + c1.abs() + (h * c2).abs()))
    if dresidual is not None:
        dx = dx + dresidual
    err = err + 4 * U * dx.abs() + ROUND[dtype] * dx.abs() * (1 + ROUND[dtype]) + TINY
    dgamma, dbeta = (dy * h).sum(0), dy.sum(0)
    # a workgroup's rows one after the other, then the workgroups
    m = (rows / 256 + 64) * U
    y = h * gamma + beta
    ey = 8 * U * (y.abs() + beta.abs()) + ROUND[dtype] * y.abs() * (1 + ROUND[dtype]) + TINY
    return (dx, dgamma, dbeta, y), (err, (m + 4 * U) * (dy * h).abs().sum(0) + TINY,
                                    m * dy.abs().sum(0) + TINY, ey)


# --------------------------------------------------------------------------
# GELU
# --------------------------------------------------------------------------
def gelu(u, da, dtype):
    """a, du in float64, and the bounds of their errors: the tail's polynomial
    is within 1.5e-7 of it, its evaluation within 16 U, and the exponential's
    argument u^2 / 2, rounded twice, moves it by u^2 U."""
    p = 0.5 * torch.special.erfc(-u * 0.5 ** 0.5)
    tail = torch.minimum(p, 1 - p).clamp(min=0)
    density = torch.exp(-u * u / 2) * (0.5 / torch.pi) ** 0.5
    rel = 1.5e-7 + 16 * U + u * u * U
    ep = tail * rel + U * p
    a, slope = u * p, p + u * density
    ea = u.abs() * (ep + TINY) + 2 * U * a.abs()
    es = ep + (u * density).abs() * (rel + 4 * U) + 2 * U * slope.abs() + TINY * (1 + u.abs())
    du = da * slope
    r = ROUND[dtype] * (1 + ROUND[dtype])
    return (a, du), (ea + r * a.abs() + TINY,
                     da.abs() * es + (r + 2 * U) * du.abs() + TINY)


def weight_grad(dy, x):
    """dy^T x in float64, and the bound of a 32-bit sum in any order."""
    return dy.t() @ x, (dy.shape[0] + 8) * U * (dy.abs().t() @ x.abs()) + TINY


def check(got, want, bound, what):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), "%s: %d of %d outside, worst %g over its bound %g, first at %s" % (
        what, int(bad.sum()), bad.numel(),
        float(torch.nan_to_num((got - want).abs() / bound, nan=float("inf")).max()),
        float(bound[bad][0]), bad.nonzero()[0].tolist())
