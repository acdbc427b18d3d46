"""Plain 64-bit forms of the token operators (rotary positions, log probabilities,
moments in 8 bits) and the bounds that their kernels have to keep.

Half a step of a rounding is finfo.eps / 2: u = 2^-24 for fp32, 2^-8 for bf16.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24


def out_step(dtype):
    return torch.finfo(dtype).eps / 2


def numbers(shape, seed, dtype, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (std * torch.randn(*shape, device="cuda", generator=gen)).to(dtype)


# --------------------------------------------------------------------------
# Rotary positions
# --------------------------------------------------------------------------
def angles(positions, turns):
    """cos and sin of 2 pi positions turns, the product and the fraction of a turn in
    numpy's extended precision."""
    t = np.asarray(positions, np.longdouble)[:, None] * np.asarray(turns, np.longdouble)
    f = (t - np.rint(t)).astype(np.float64) * (2 * math.pi)
    return np.cos(f), np.sin(f), np.abs(t).astype(np.float64)


def rotated(x, positions, turns, interleaved, scale, backward):
    """x [tokens, groups, heads, dim] in 64 bits, rotated; and a bound on a kernel's error
    before its result is rounded to a type.

    cos and sin in fp32: the angle's rounding (up to pi / 4: u / 2) and the polynomial's last
    step (u / 2) and inner ones (their sum is below 0.3 with about three roundings) are below
    2 u together; the product with the scale adds u, the two products and their sum 2 u more.
    The angle's product in 64 bits is off by 2^-53 of itself, in turns."""
    n = 2 * len(turns)
    c, s, t = (torch.from_numpy(a).to(x.device)[:, None, None, :]
               for a in angles(positions.cpu().numpy(), turns.cpu().numpy()))
    x = x.double()
    first = (..., slice(0, n, 2)) if interleaved else (..., slice(0, n // 2))
    second = (..., slice(1, n, 2)) if interleaved else (..., slice(n // 2, n))
    if backward:
        s = -s
    a, b = x[first], x[second]
    want, bound = x.clone(), torch.zeros_like(x)
    want[first] = scale * (a * c - b * s)
    want[second] = scale * (a * s + b * c)
    off = abs(scale) * (a.abs() + b.abs()) * (5 * U + 2 * math.pi * 2.0 ** -53 * t)
    bound[first] = off
    bound[second] = off
    return want, bound


# --------------------------------------------------------------------------
# Log probabilities
# --------------------------------------------------------------------------
def softmax_parts(x):
    """lse, ln S, entropy and mean distance E|d| from the maximum, in 64 bits."""
    x = x.double()
    top = x.amax(1, keepdim=True)
    d = torch.where(torch.isinf(x), torch.full_like(x, -1e9), x - top)
    e = torch.exp(d)
    s = e.sum(1)
    w = (e * d).sum(1)
    ln = torch.log(s)
    return top[:, 0] + ln, ln, ln - w / s, -w / s


def sum_bound(vocab, mean_d):
    """Relative error of the kernel's S, and of W's terms beside it.

    An element's e: its distance d is rounded (|d| u), multiplied by log2 e (|d| u, and the
    constant's own 0.3 |d| u), and the exponential is within a unit in the last place (2 u);
    rescaling to a joint maximum splits d, no more.  A lane adds 8 values, then at least 64 lanes
    share the row: vocab / 512 partial sums one after the other, each with a rescaling
    (3 u for its factor and product); 6 steps in a wave, and slices and waves: fewer than 40."""
    return U * (2.4 * mean_d + 2 + 8 + 4 * math.ceil(vocab / 512) + 40)


def forward_bounds(vocab, lse, ln, h, mean_d, lp):
    rel = sum_bound(vocab, mean_d)
    log = 2 * U * ln.abs() + 2 * U           # logf, within a unit; near 1 of its terms
    b_lse = rel + log + 2 * U * lse.abs()
    b_lp = rel + log + 2 * U * lp.abs()
    b_h = rel + log + (2 * rel + 4 * U) * mean_d + 2 * U * h.abs()
    return b_lse, b_lp, b_h


def gradient(x, targets, lse, g, h=None, entropy=None, rel_s=None):
    """dx in 64 bits from lse (what the kernel is given, or its own with a relative error rel_s
    of S) and the bound of its error before the last rounding: d and d - ln rounded and
    multiplied (3.4 |d| u), the exponential 2 u, the factor's three terms u each, a product."""
    x = x.double()
    valid = (targets >= 0)
    g = torch.where(valid, g.double(), torch.zeros_like(lse))
    logs = (x - lse[:, None]).clamp(min=-1e4)
    p = torch.exp(x - lse[:, None])
    c = -g[:, None].expand_as(x)
    size = g.abs()[:, None].expand_as(x)
    if h is not None:
        c = c - h.double()[:, None] * (logs + entropy[:, None])
        size = size + h.double().abs()[:, None] * (logs.abs() + entropy.abs()[:, None] + lse.abs()[:, None])
    want = p * c
    rel = (3.4 * logs.abs() + 2 * lse.abs()[:, None] + 4) * U
    if rel_s is not None:
        rel = rel + rel_s[:, None]
    bound = p * (rel * c.abs() + 5 * U * size) + 1e-37
    # the exponential has no results below the normal numbers: relative to the largest logit
    # or to lse, whose sum is 1 or more, e^d < 2^-126 counts as 0, and then p |c| is missing,
    # which is below 2^-126 |c| (|c| is past 8, and this past 1e-37, where h is not 0 and
    # log p is near -87)
    bound = bound + torch.where(p < 2.0 ** -125, 2.0 ** -126 * c.abs(), torch.zeros_like(p))
    if rel_s is not None and h is not None:
        bound = bound + p * h.double().abs()[:, None] * (2 * rel_s * (1 + entropy.abs()))[:, None]
    rows = torch.arange(x.shape[0], device=x.device)
    at = targets.clamp(min=0)
    want[rows, at] += g
    bound = bound + U * want.abs()
    return want, bound


def top_ids(x, k):
    """The k largest of each row, the lower of equals first (stable, both zeros one)."""
    return torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :k]


# --------------------------------------------------------------------------
# Moments in 8 bits, numpy, every operation rounded to fp32 as the format says
# --------------------------------------------------------------------------
BLOCK = 256
f32 = np.float32


def _blocks(x):
    n = len(x)
    pad = np.zeros((-(-n // BLOCK) * BLOCK,), f32)
    pad[:n] = x
    return pad.reshape(-1, BLOCK)


def encode_state(x, moment):
    with np.errstate(all="ignore"):
        y = _blocks(x)
        if moment == 2:
            y = np.sqrt(y)
        bad = ~np.isfinite(y).all(1)
        top = np.abs(np.where(np.isfinite(y), y, 0)).max(1).astype(f32)
        whole = f32(127 if moment == 1 else 65025)
        held = (top >= f32(2.0 ** -100)) if moment == 1 else (top > 0)
        scale = np.where(held, top / whole, f32(0)).astype(f32)
        inv = np.where(held, whole / top, f32(0)).astype(f32)
        t = (np.where(np.isfinite(y), y, 0).astype(f32) * inv[:, None]).astype(f32)
        if moment == 1:
            codes = np.rint(t)
        else:
            t = t.astype(np.float64)
            codes = np.floor(np.sqrt(t) + 0.5)
            codes = np.where((codes > 0) & ((codes - 0.5) ** 2 > t), codes - 1, codes)
            codes = np.where((codes + 0.5) ** 2 <= t, codes + 1, codes)
            codes = np.where((y > 0) & (codes < 1), 1, codes)
        codes[bad | ~held] = 0
        scale[bad] = np.nan
    dtype = np.int8 if moment == 1 else np.uint8
    return codes.astype(dtype).reshape(-1)[:len(x)], scale


def decode_state(codes, scale, moment):
    with np.errstate(all="ignore"):
        c = codes.astype(f32)
        s = np.repeat(scale, BLOCK)[:len(c)]
        if moment == 1:
            return c * s
        r = (c * c) * s
        return r * r
