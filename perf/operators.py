"""Timed cases of the layer operators: layer norm's forward and backward pass,
GELU's, activation checkpoints in 8 bits, and a linear layer's weight gradient,
each one pass through the public calls of `paper_2407_01614_amd.zpp` (`own`) or
the same in elementary torch operations in 32 bits.

A case is a dict: `op` names what runs, `rows` the tokens, `cols` the features
of a token (for the weight gradient: `n` features of the output gradient and
`k` of the input), `type` the matrices' element type ("bf16" or "f32"),
`params` the type of layer norm's weight and bias, `saved` what the backward
pass reads ("i8" a checkpoint in 8 bits, or the matrices' own type), `pad` how
many features the matrices' rows lie further apart than they are long (a slice
of a wider buffer), and the optional operands.  Feature sizes are those of the
Falcon layers of `workloads.py` (hidden 4544 with 18176 in the MLP and 4672 out
of the fused query-key-value product, hidden 8192 with 32768), or generic.

A checkpoint holds blocks of 64 consecutive features of a token as int8 codes
with a power of two as their scale: the smallest 2^e, e >= -126, that keeps the
block's largest magnitude within 127.
"""
import torch

own = False

BLOCK = 64
EPS = 1e-5
# activations with some channels far larger than the others, as decoder layers
# have them; gradients of activations; weights around one and biases around zero
ACT_STD, OUTLIER_STD, OUTLIER_EVERY, GRAD_STD, PARAM_STD = 1.0, 20.0, 512, 1e-3, 0.1

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # layer norm of a single token, as it is answered
        dict(name="norm-fwd-token", op="norm_forward", rows=1, cols=4544, type="bf16",
             params="bf16", saved="bf16", pad=0, residual=False),
        # layer norm's backward pass in 32 bits on a small odd model, saved as it was
        dict(name="norm-bwd-f32-odd", op="norm_backward", rows=1000, cols=1153, type="f32",
             params="f32", saved="f32", pad=3, residual=False, recompute=False),
        # backward of a Falcon-7B layer's norm from the 8-bit checkpoint of its
        # input, with the residual branch's gradient, giving back the normalised
        # output that the next linear layer's weight gradient takes
        dict(name="norm-bwd-7b", op="norm_backward", rows=4096, cols=4544, type="bf16",
             params="bf16", saved="i8", pad=0, residual=True, recompute=True),
        # both passes of a Falcon-40B layer's norm over a long batch: the residual
        # added and the 8-bit checkpoint written going forward, read going back
        dict(name="norm-train-40b", op="norm_train", rows=8192, cols=8192, type="bf16",
             params="f32", saved="i8", pad=0, residual=True, recompute=False),
        # GELU of a short ragged batch in 32 bits, nothing saved
        dict(name="gelu-fwd-f32-short", op="gelu_forward", rows=33, cols=18176, type="f32",
             saved="f32", pad=0),
        # GELU's backward pass in a Falcon-7B layer from the 8-bit checkpoint of its
        # input, giving back its output for the second linear layer's weight gradient
        dict(name="gelu-bwd-7b", op="gelu_backward", rows=4096, cols=18176, type="bf16",
             saved="i8", pad=0, recompute=True),
        # both passes in a Falcon-40B layer through the 8-bit checkpoint
        dict(name="gelu-train-40b", op="gelu_train", rows=2048, cols=32768, type="bf16",
             saved="i8", pad=0, recompute=False),
        # one layer's input saved in 8 bits and read back: a small odd one in 32
        # bits, and a long one
        dict(name="checkpoint-f32-odd", op="checkpoint", rows=129, cols=1001, type="f32",
             saved="i8", pad=7),
        dict(name="checkpoint-40b", op="checkpoint", rows=8192, cols=8192, type="bf16",
             saved="i8", pad=0),
        # weight gradient of a small odd linear layer from its bf16 input
        dict(name="wgrad-small-odd", op="weight_grad", rows=77, n=1000, k=777, type="bf16",
             saved="bf16", pad=1),
        # of Falcon-7B's fused query-key-value product, a ragged batch, the
        # input's 8-bit checkpoint
        dict(name="wgrad-qkv-7b", op="weight_grad", rows=2047, n=4672, k=4544, type="bf16",
             saved="i8", pad=0),
        # of Falcon-7B's first MLP product from the input's 8-bit checkpoint
        dict(name="wgrad-mlp-7b", op="weight_grad", rows=4096, n=18176, k=4544, type="bf16",
             saved="i8", pad=0),
    ]


MOST_ELEMENTS = 8192 * 8192
MOST_PRODUCTS = 4096 * 18176 * 4544


def _log_size(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["norm_forward", "norm_backward", "norm_train", "gelu_forward",
                     "gelu_backward", "gelu_train", "checkpoint", "weight_grad", "weight_grad"])
    c = dict(op=op, type=rng.choice(["bf16", "bf16", "f32"]), pad=rng.choice([0, 0, 1, 8, 131]))
    if op == "weight_grad":
        c["type"] = "bf16"
        c["saved"] = rng.choice(["bf16", "i8"])
        while True:
            c["rows"] = _log_size(rng, 1, 8192)
            c["n"] = _log_size(rng, 64, 18176)
            c["k"] = _log_size(rng, 64, 8192)
            if rng.random() < 0.5:
                c["n"], c["k"] = (-(-x // 64) * 64 for x in (c["n"], c["k"]))
            if c["rows"] * c["n"] * c["k"] <= MOST_PRODUCTS:
                return c
    wide = 32768 if op.startswith("gelu") else 16384
    while True:
        c["rows"] = _log_size(rng, 1, 16384)
        c["cols"] = _log_size(rng, 64, wide)
        if rng.random() < 0.5:
            c["cols"] = -(-c["cols"] // 64) * 64
        if c["rows"] * c["cols"] <= MOST_ELEMENTS:
            break
    if op in ("norm_train", "gelu_train", "checkpoint"):
        c["saved"] = "i8"
    elif op.endswith("forward"):
        c["saved"] = c["type"]
    else:
        c["saved"] = rng.choice([c["type"], "i8"])
    if op.startswith("norm"):
        c["params"] = rng.choice(["bf16", "f32"])
        c["residual"] = rng.random() < 0.5
    if op.endswith("backward") or op.endswith("train"):
        c["recompute"] = rng.random() < 0.5
    return c


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def _matrix(rows, cols, pad, dtype):
    """A matrix [rows, cols] of undefined values, a slice of a buffer `pad` wider."""
    return torch.empty(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def _normal(gen, rows, cols, pad, dtype, std):
    m = _matrix(rows, cols, pad, dtype)
    m.copy_(torch.randn(rows, cols, device="cuda", generator=gen) * std)
    return m


def _activations(gen, rows, cols, pad, dtype):
    std = torch.full((cols,), ACT_STD, device="cuda")
    std[OUTLIER_EVERY // 3::OUTLIER_EVERY] = OUTLIER_STD
    return _normal(gen, rows, cols, pad, dtype, std)


def _empty_checkpoint(rows, cols):
    return (torch.empty(rows, cols, dtype=torch.int8, device="cuda"),
            torch.empty(rows, -(-cols // BLOCK), dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, dtype, pad, rows = case["op"], TYPES[case["type"]], case["pad"], case["rows"]
    s = dict(case=case)
    if op == "weight_grad":
        n, k = case["n"], case["k"]
        s["dy"] = _normal(gen, rows, n, pad, dtype, GRAD_STD)
        x = _activations(gen, rows, k, pad, dtype)
        s["x"] = _encode(x.float()) if case["saved"] == "i8" else x
        s["dw"] = torch.empty(n, k, dtype=torch.float32, device="cuda")
        return s
    cols = case["cols"]
    s["x"] = _activations(gen, rows, cols, pad, dtype)
    if op == "checkpoint":
        s["saved"] = _empty_checkpoint(rows, cols)
        s["out"] = _matrix(rows, cols, pad, dtype)
        return s
    forward = not op.endswith("backward")
    backward = not op.endswith("forward")
    s["y"] = _matrix(rows, cols, pad, dtype) if forward or case["recompute"] else None
    if op.startswith("norm"):
        weights = TYPES[case["params"]]
        s["gamma"] = (1 + PARAM_STD * torch.randn(cols, device="cuda", generator=gen)).to(weights)
        s["beta"] = (PARAM_STD * torch.randn(cols, device="cuda", generator=gen)).to(weights)
        s["mean"] = torch.empty(rows, device="cuda")
        s["rstd"] = torch.empty(rows, device="cuda")
        if forward and case["residual"]:
            s["residual"] = _activations(gen, rows, cols, pad, dtype)
            s["total"] = _matrix(rows, cols, pad, dtype)
        if backward:
            s["dgamma"] = torch.empty(cols, device="cuda")
            s["dbeta"] = torch.empty(cols, device="cuda")
            if case["residual"]:
                s["dresidual"] = _normal(gen, rows, cols, pad, dtype, GRAD_STD)
        if not forward:
            s["mean"], s["rstd"] = _statistics(s["x"].float())
    if backward:
        s["dy"] = _normal(gen, rows, cols, pad, dtype, GRAD_STD)
        s["dx"] = _matrix(rows, cols, pad, dtype)
        if forward:
            s["saved"] = _empty_checkpoint(rows, cols)
            s["again"] = _matrix(rows, cols, pad, dtype) if case["recompute"] else None
        elif case["saved"] == "i8":
            s["x"] = _encode(s["x"].float())
    return s


# --------------------------------------------------------------------------
# The plain forms, in 32 bits
# --------------------------------------------------------------------------
def _power_of_two(e):
    return ((e + 127) << 23).view(torch.float32)


def _encode(x):
    """Codes and biased scale exponents of a float32 matrix."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    top = x.abs().amax(2)
    part, e = torch.frexp(top)          # top = part * 2^e, 1/2 <= part < 1
    e = (e - 7 + (part > 127 / 128).int()).clamp(min=-126)
    e = torch.where(top == 0, torch.full_like(e, -126), e)
    most = torch.where(e >= 122, 63.0, 127.0)[:, :, None]   # what stays finite
    codes = torch.round(x * _power_of_two(-e)[:, :, None])
    codes = torch.maximum(torch.minimum(codes, most), -most)
    finite = torch.isfinite(top)
    codes = torch.where(finite[:, :, None], codes, torch.zeros_like(codes))
    exps = torch.where(finite, e + 127, torch.full_like(e, 255))
    return (codes.to(torch.int8).view(rows, blocks * BLOCK)[:, :cols].contiguous(),
            exps.to(torch.uint8))


def _decode(saved):
    """The float32 values of a checkpoint."""
    codes, exps = saved
    scale = (exps.int() << 23).view(torch.float32)
    scale = torch.where(exps == 255, torch.full_like(scale, float("nan")), scale)
    return codes.float() * scale.repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def _values(x):
    return _decode(x) if isinstance(x, tuple) else x.float()


def _statistics(x):
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, torch.rsqrt(var + EPS)


def _plain_norm_forward(x, gamma, beta):
    mean, rstd = _statistics(x)
    return (x - mean[:, None]) * rstd[:, None] * gamma.float() + beta.float(), mean, rstd


def _plain_norm_backward(dy, x, gamma, beta, mean, rstd, dresidual):
    dy, gamma = dy.float(), gamma.float()
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if dresidual is not None:
        dx = dx + dresidual.float()
    return dx, (dy * xh).sum(0), dy.sum(0), xh * gamma + beta.float()


def _plain_cdf(u):
    return 0.5 * (1 + torch.erf(u * 0.7071067811865476))


def _plain_gelu_backward(da, u):
    p = _plain_cdf(u)
    density = torch.exp(-0.5 * u * u) * 0.3989422804014327
    return da.float() * (p + u * density), u * p


def _run_plain(s):
    case = s["case"]
    op, dtype = case["op"], TYPES[case["type"]]
    out = {}
    if op == "weight_grad":
        out["dw"] = s["dy"].float().t() @ _values(s["x"])
    elif op == "checkpoint":
        out["values"] = _decode(_encode(s["x"].float())).to(dtype)
    elif op.startswith("norm"):
        x, mean, rstd = s["x"], s["mean"], s["rstd"]
        if op != "norm_backward":
            if case["residual"]:
                x = (x.float() + s["residual"].float()).to(dtype)
                out["total"] = x
            y, mean, rstd = _plain_norm_forward(x.float(), s["gamma"], s["beta"])
            out.update(y=y.to(dtype), mean=mean, rstd=rstd)
        if op != "norm_forward":
            seen = _decode(_encode(x.float())) if op == "norm_train" else _values(x)
            dx, dgamma, dbeta, again = _plain_norm_backward(s["dy"], seen, s["gamma"], s["beta"],
                                                            mean, rstd, s.get("dresidual"))
            out.update(dx=dx.to(dtype), dgamma=dgamma, dbeta=dbeta)
            if case["recompute"]:
                out["again"] = again.to(dtype)
    else:
        x = s["x"]
        if op != "gelu_backward":
            u = x.float()
            out["a"] = (u * _plain_cdf(u)).to(dtype)
        if op != "gelu_forward":
            seen = _decode(_encode(x.float())) if op == "gelu_train" else _values(x)
            du, again = _plain_gelu_backward(s["dy"], seen)
            out["du"] = du.to(dtype)
            if case["recompute"]:
                out["again"] = again.to(dtype)
    return out


# --------------------------------------------------------------------------
# The framework's calls
# --------------------------------------------------------------------------
def _workspace(s, nbytes):
    """The program's workspace: laid out on its first pass, then kept."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _run_own(s):
    from paper_2407_01614_amd import zpp
    case = s["case"]
    op, rows = case["op"], case["rows"]
    if op == "weight_grad":
        ws = _workspace(s, zpp.weight_grad_workspace(rows, case["n"], case["k"]))
        zpp.weight_grad(s["dy"], s["x"], s["dw"], ws)
        return dict(dw=s["dw"])
    if op == "checkpoint":
        zpp.checkpoint_save(s["x"], s["saved"])
        zpp.checkpoint_load(s["saved"], s["out"])
        return dict(values=s["out"])
    out = {}
    x, again = s["x"], s["y"]
    if op.startswith("norm"):
        if op != "norm_backward":
            zpp.layer_norm_forward(x, s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"],
                                   eps=EPS, residual=s.get("residual"), total=s.get("total"),
                                   saved=s.get("saved"))
            out.update(y=s["y"], mean=s["mean"], rstd=s["rstd"])
            if case["residual"]:
                out["total"] = s["total"]
            x, again = s.get("saved"), s.get("again")
        if op != "norm_forward":
            ws = _workspace(s, zpp.layer_norm_backward_workspace(rows, case["cols"]))
            zpp.layer_norm_backward(s["dy"], x, s["gamma"], s["mean"], s["rstd"], s["dx"],
                                    s["dgamma"], s["dbeta"], ws, dresidual=s.get("dresidual"),
                                    beta=s["beta"] if case["recompute"] else None, y=again)
            out.update(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
            if case["recompute"]:
                out["again"] = again
        return out
    if op != "gelu_backward":
        zpp.gelu_forward(x, s["y"], saved=s.get("saved"))
        out["a"] = s["y"]
        x, again = s.get("saved"), s.get("again")
    if op != "gelu_forward":
        zpp.gelu_backward(s["dy"], x, s["dx"], a=again)
        out["du"] = s["dx"]
        if case["recompute"]:
            out["again"] = again
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# --------------------------------------------------------------------------
def work(case):
    op, rows = case["op"], case["rows"]
    size = {"bf16": 2, "f32": 4}[case["type"]]
    if op == "weight_grad":
        n, k = case["n"], case["k"]
        x = rows * (k + -(-k // BLOCK)) if case["saved"] == "i8" else 2 * rows * k
        return dict(bytes=2 * rows * n + x + 4 * n * k, flops=2 * rows * n * k)
    cols = case["cols"]
    whole, saved = rows * cols * size, rows * (cols + -(-cols // BLOCK))
    if op == "checkpoint":
        return dict(bytes=2 * whole + 2 * saved, flops=4 * rows * cols)
    moved, flops = 0, 0
    if not op.endswith("backward"):
        moved += 2 * whole + (saved if op.endswith("train") else 0)
        flops += 8 * rows * cols
    if not op.endswith("forward"):
        moved += 2 * whole + (saved if case["saved"] == "i8" else whole)
        moved += whole if case["recompute"] else 0
        flops += 12 * rows * cols
    if op.startswith("norm"):
        width = {"bf16": 2, "f32": 4}[case["params"]]
        if not op.endswith("backward"):
            moved += (2 * whole if case["residual"] else 0) + 8 * rows + 2 * width * cols
        if not op.endswith("forward"):
            moved += (whole if case["residual"] else 0) + 8 * rows + (width + 8) * cols
            moved += width * cols if case["recompute"] else 0
    return dict(bytes=moved, flops=flops)


def _exact_power(e):
    """2^e in 64 bits, by its bits (the device's ldexp is off in the last of them)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_saved(x):
    """A checkpoint's values in 64 bits, from the definition: every block of a
    row over the smallest power of two that keeps it within 127."""
    rows, cols = x.shape
    values = torch.empty_like(x)
    for at in range(0, cols, BLOCK):
        part = x[:, at:at + BLOCK]
        top = part.abs().amax(1, keepdim=True)
        step = torch.full_like(top, 2.0 ** -126)
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140))).clamp(min=-126)
        for down in (7, 6, 5):  # the largest of the three that still is too small, doubled
            less = _exact_power(e - down)
            step = torch.where((127 * less < top) & (2 * less > step), 2 * less, step)
        most = torch.where(step < 2.0 ** 122, 127.0, 63.0)  # a code's value is a finite float
        values[:, at:at + BLOCK] = torch.round(part / step).clamp(-most, most) * step
    return values


def _exact_values(x):
    if not isinstance(x, tuple):
        return x.double()
    codes, exps = x
    at = torch.arange(codes.shape[1], device=codes.device) // BLOCK
    return codes.double() * _exact_power(exps.double()[:, at] - 127)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "weight_grad":
        return dict(dw=torch.matmul(s["dy"].double().t().contiguous(), _exact_values(s["x"])))
    if op == "checkpoint":
        return dict(values=_exact_saved(s["x"].double()))
    out = {}
    dtype = TYPES[case["type"]]
    x = None if isinstance(s["x"], tuple) else s["x"].double()
    if op.startswith("norm"):
        mean, rstd = s["mean"].double(), s["rstd"].double()
        gamma, beta = s["gamma"].double(), s["beta"].double()
        if op != "norm_backward":
            if case["residual"]:
                x = (x + s["residual"].double()).to(dtype).double()
                out["total"] = x
            var, mean = torch.var_mean(x, dim=1, unbiased=False)
            rstd = (var + EPS).pow(-0.5)
            out.update(y=torch.addcmul(beta, (x - mean[:, None]) * rstd[:, None], gamma),
                       mean=mean, rstd=rstd)
        if op != "norm_forward":
            seen = _exact_saved(x) if op == "norm_train" else _exact_values(s["x"])
            dy, cols = s["dy"].double(), case["cols"]
            z = (seen - mean[:, None]) * rstd[:, None]
            weighted = dy * gamma
            c1 = weighted.sum(1, keepdim=True) / cols
            c2 = (weighted * z).sum(1, keepdim=True) / cols
            dx = (weighted - c1 - z * c2) * rstd[:, None]
            if "dresidual" in s:
                dx += s["dresidual"].double()
            out.update(dx=dx, dgamma=(dy * z).sum(0), dbeta=dy.sum(0))
            if case["recompute"]:
                out["again"] = torch.addcmul(beta, z, gamma)
        return out

    def cdf(u):
        return 0.5 * torch.special.erfc(-u * 0.5 ** 0.5)

    if op != "gelu_backward":
        out["a"] = x * cdf(x)
    if op != "gelu_forward":
        u = _exact_saved(x) if op == "gelu_train" else _exact_values(s["x"])
        density = torch.exp(-u * u / 2) * (0.5 / torch.pi) ** 0.5
        out["du"] = s["dy"].double() * (cdf(u) + u * density)
        if case["recompute"]:
            out["again"] = u * cdf(u)
    return out
