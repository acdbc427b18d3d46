"""Timed cases of the operators of a token model's training step: rotary positions,
log probabilities with their gradient, and AdamW over many tensors with its moments
in 32 or in 8 bits; each one pass through the public calls of
`paper_2407_01614_amd.zpp` (`own`) or the same in elementary torch operations.

A case is a dict; `op` names what runs.  Sizes are those of the Llama-2 and Falcon
layers of `workloads.py`, or generic.

Rotary: `tokens` of `heads` query heads and `kv_heads` key heads of `dim` features,
the first `rotated` of which turn, as halves or as neighbours (`interleaved`).
`layout`: "separate" query and key arrays, rotated into others; "fused", the columns
of one buffer with the values, rotated in place; "grouped", the same with every key
head next to its queries.  `far`: the last position.  `linear`: positions are divided by it.
`scale`: a factor on what is rotated.  `way`: forward, backward or both.

Log probabilities: `rows` of `vocab` logits.  `way`: "forward", "backward" (from the
forward pass's sums) or "train" (both in one call).  `entropy`: with the entropy and
its gradient.  `top`: so many most probable tokens.  `pad`: how many logits the rows
lie further apart than they are long.

AdamW: `sizes` the tensors' lengths ("4096*65": 65 of them), `states` the moments' type,
`grad` the gradients'.  With moments in 8 bits the pass ends with their export to 32.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # queries and key of one new token of Falcon-7B, in place in the fused product's output
        dict(name="rotary-token", op="rotary", tokens=1, heads=71, kv_heads=1, dim=64, rotated=64,
             layout="fused", interleaved=False, type="bf16", far=2047, linear=1.0, scale=1.0,
             way="forward"),
        # part of an odd head in 32 bits, neighbours as pairs, far positions, scaled
        dict(name="rotary-f32-odd", op="rotary", tokens=333, heads=5, kv_heads=5, dim=80,
             rotated=20, layout="separate", interleaved=True, type="f32", far=1000000, linear=8.0,
             scale=1.125, way="forward"),
        # a Llama-2-7B layer's queries and keys, forward
        dict(name="rotary-7b", op="rotary", tokens=4096, heads=32, kv_heads=32, dim=128,
             rotated=128, layout="separate", interleaved=True, type="bf16", far=4095, linear=1.0,
             scale=1.0, way="forward"),
        # a Falcon-40B layer's: both passes in place in the fused product's output, whose
        # eight keys lie behind their sixteen queries each; positions for a longer context
        dict(name="rotary-train-40b", op="rotary", tokens=8192, heads=128, kv_heads=8, dim=64,
             rotated=64, layout="grouped", interleaved=False, type="bf16", far=8191, linear=4.0,
             scale=1.0, way="both"),
        # a new token's log probability with entropy and the twenty best, Falcon's vocabulary
        dict(name="logprobs-token", op="log_probs", rows=1, vocab=65024, type="bf16", pad=0,
             entropy=True, top=20, way="forward"),
        # a short ragged batch in 32 bits over an odd vocabulary, five best
        dict(name="logprobs-f32-odd", op="log_probs", rows=77, vocab=32003, type="f32", pad=5,
             entropy=False, top=5, way="forward"),
        # log probabilities and entropies of a batch, Falcon's vocabulary
        dict(name="logprobs-fwd-40b", op="log_probs", rows=8192, vocab=65024, type="bf16", pad=0,
             entropy=True, top=0, way="forward"),
        # the gradient of log probabilities and entropies, Llama-2's vocabulary
        dict(name="logprobs-bwd-7b", op="log_probs", rows=4096, vocab=32000, type="bf16", pad=0,
             entropy=True, top=0, way="backward"),
        # the loss of a training step and its gradient, Falcon's vocabulary
        dict(name="logprobs-train-40b", op="log_probs", rows=4096, vocab=65024, type="bf16", pad=0,
             entropy=False, top=0, way="train"),
        # the norms' weights of Llama-2-7B: many small tensors, bf16 gradients
        dict(name="adam-norms", op="adam", sizes="4096*65", states="f32", grad="bf16"),
        # a Llama-2-7B layer, moments in 32 bits
        dict(name="adam-f32-7b", op="adam", sizes="16777216*4,45088768*3,4096*2", states="f32",
             grad="f32"),
        # a Falcon-7B layer, moments in 8 bits
        dict(name="adam-i8-7b", op="adam", sizes="21229568,20647936,82591744*2,4544*2",
             states="i8", grad="f32"),
    ]


MOST_ROTARY_BYTES = 2 * 8192 * 136 * 64 * 2
MOST_LOGITS_BYTES = 8192 * 65024 * 2
MOST_ADAM = 202403840


def _log_size(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _draw_rotary(rng):
    c = dict(op="rotary", type=rng.choice(["bf16", "bf16", "f32"]), interleaved=rng.random() < 0.5,
             layout=rng.choice(["separate", "fused", "grouped"]), scale=1.0,
             way=rng.choice(["forward", "backward", "both"]))
    size = 4 if c["type"] == "f32" else 2
    while True:
        c["tokens"] = _log_size(rng, 1, 16384)
        c["kv_heads"] = _log_size(rng, 1, 32)
        c["heads"] = c["kv_heads"] * _log_size(rng, 1, 32)
        c["dim"] = rng.choice([64, 128, 256, 2 * _log_size(rng, 1, 160)])
        heads = c["heads"] + c["kv_heads"]
        moved = 2 * c["tokens"] * heads * c["dim"] * size * (2 if c["way"] == "both" else 1)
        if c["heads"] <= 128 and moved <= 2 * MOST_ROTARY_BYTES:
            break
    c["rotated"] = c["dim"] if rng.random() < 0.6 else 2 * rng.randint(1, c["dim"] // 2)
    c["far"] = _log_size(rng, c["tokens"], 4000000)
    c["linear"] = rng.choice([1.0, 1.0, 2.0, 8.0])
    if c["layout"] == "separate" and c["way"] != "both":
        c["scale"] = rng.choice([1.0, 1.25])
    return c


def _draw_log_probs(rng):
    c = dict(op="log_probs", type=rng.choice(["bf16", "bf16", "f32"]),
             way=rng.choice(["forward", "forward", "backward", "train"]),
             entropy=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 8, 131]), top=0)
    size = (4 if c["type"] == "f32" else 2) * (1 if c["way"] == "forward" else 2)
    while True:
        c["rows"] = _log_size(rng, 1, 16384)
        c["vocab"] = _log_size(rng, 16, 262144)
        if rng.random() < 0.5:
            c["vocab"] = -(-c["vocab"] // 64) * 64
        if c["rows"] * c["vocab"] * size <= MOST_LOGITS_BYTES:
            break
    if c["way"] == "forward" and c["rows"] * c["vocab"] <= 1 << 26:
        c["top"] = rng.choice([0, 1, 5, 20, 32])
        c["top"] = min(c["top"], c["vocab"])
    return c


def _draw_adam(rng):
    c = dict(op="adam", states=rng.choice(["f32", "i8", "i8"]), grad=rng.choice(["f32", "bf16"]))
    left, parts = _log_size(rng, 1 << 10, MOST_ADAM), []
    for _ in range(rng.randint(1, 8)):
        n = min(left, _log_size(rng, 1, 1 << 26))
        times = max(1, min(left // max(n, 1), _log_size(rng, 1, 64)))
        if n and n * times <= left:
            parts.append("%d*%d" % (n, times))
            left -= n * times
    c["sizes"] = ",".join(parts)
    return c


def draw(rng):
    return rng.choice([_draw_rotary, _draw_log_probs, _draw_log_probs, _draw_adam])(rng)


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
BASE = 10000.0
GRAD_STD = 1e-3
IGNORED = -100          # the target of a row that takes no part in the loss
BLOCK = 256             # values of a block of moments in 8 bits
LR, BETA1, BETA2, EPS, STEP, DECAY = 1e-4, 0.9, 0.95, 1e-8, 10, 0.1


def _turns(rotated, linear):
    """Turns (of 2 pi) a position of each pair."""
    at = torch.arange(rotated // 2, dtype=torch.float64, device="cuda")
    return BASE ** (-2 * at / rotated) / (2 * math.pi * linear)


def _prepare_rotary(case, gen):
    tokens, heads, kv, dim = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    s = dict(turns=_turns(case["rotated"], case["linear"]))
    s["positions"] = torch.arange(case["far"] + 1 - tokens, case["far"] + 1, device="cuda")

    def array(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(TYPES[case["type"]])

    if case["layout"] == "separate":
        s["x"], s["k"] = array(tokens, 1, heads, dim), array(tokens, 1, kv, dim)
        s["out"], s["k_out"] = torch.empty_like(s["x"]), torch.empty_like(s["k"])
        return s
    # the values' heads lie behind the keys' and stay as they are
    groups = kv if case["layout"] == "grouped" else 1
    turning = (heads + kv) // groups
    s["buffer"] = array(tokens, groups, turning + kv // groups, dim)
    s["x"] = s["out"] = s["buffer"][:, :, :turning]
    s["k"] = s["k_out"] = None
    return s


def _prepare_log_probs(case, gen):
    rows, vocab, dtype = case["rows"], case["vocab"], TYPES[case["type"]]

    def logits():
        return torch.empty(rows, vocab + case["pad"], dtype=dtype, device="cuda")[:, :vocab]

    s = dict(x=logits())
    masked = vocab // 64
    targets = torch.randint(vocab - masked, (rows,), device="cuda", generator=gen)
    # logits of a model that has learned something: the right token stands out by some
    # amount, and a stretch of the vocabulary is masked
    s["x"].copy_(2 * torch.randn(rows, vocab, device="cuda", generator=gen))
    at = targets[:, None]
    s["x"].scatter_add_(1, at, (6 * torch.rand(rows, 1, device="cuda", generator=gen)).to(dtype))
    s["x"][:, vocab - masked:] = float("-inf")
    skipped = torch.rand(rows, device="cuda", generator=gen) < 1 / 16
    s["targets"] = torch.where(skipped, torch.full_like(targets, IGNORED), targets)
    for name in ("log_probs", "lse", "entropies"):
        s[name] = torch.empty(rows, device="cuda")
    if case["way"] == "backward":
        fine = s["x"].double()
        s["lse"] = torch.logsumexp(fine, 1).float()
        s["entropies"] = _exact_entropy(fine).float()
    if case["way"] != "forward":
        s["dlog_probs"] = -torch.rand(rows, device="cuda", generator=gen) / rows
        if case["entropy"]:
            s["dentropies"] = torch.randn(rows, device="cuda", generator=gen) * (0.01 / rows)
        s["dx"] = logits()
    if case["top"]:
        s["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
        s["top_log_probs"] = torch.empty(rows, case["top"], device="cuda")
    return s


def _lengths(case):
    found = []
    for part in case["sizes"].split(","):
        n, _, times = part.partition("*")
        found += [int(n)] * int(times or 1)
    return found


def _prepare_adam(case, gen):
    # the tensors are pieces of flat arrays, each from a block's first value on, as a
    # rank's partition holds them; what lies between them is zero and stays so
    lengths = _lengths(case)
    starts, end = [], 0
    for n in lengths:
        starts.append(end)
        end += -(-n // BLOCK) * BLOCK
    whole = torch.tensor(lengths, device="cuda")
    blocks = -(-whole // BLOCK)
    place = torch.arange(end // BLOCK, device="cuda") - torch.repeat_interleave(
        blocks.cumsum(0) - blocks, blocks)
    held = (torch.repeat_interleave(whole, blocks) - place * BLOCK).clamp(max=BLOCK)
    inside = torch.arange(BLOCK, device="cuda") < held[:, None]
    # weights decay, norms' and biases' tensors (the short ones) do not
    decays = [DECAY if n > 65536 else 0.0 for n in lengths]

    def flat(std):
        x = torch.randn(end // BLOCK, BLOCK, device="cuda", generator=gen)
        return x.mul_(std).mul_(inside).view(-1)

    s = dict(starts=starts, lengths=lengths, decays=decays)
    s["decay"] = torch.repeat_interleave(torch.tensor(decays, device="cuda"), blocks)[:, None]
    s["p"] = flat(0.02)
    # a gradient's rows differ in size
    rows = torch.exp2(2 * torch.randn(end // BLOCK, 1, device="cuda", generator=gen))
    s["g"] = (flat(GRAD_STD).view(-1, BLOCK) * rows).view(-1).to(TYPES[case["grad"]])
    m = (flat(GRAD_STD / 4).view(-1, BLOCK) * rows).view(-1)
    v = (flat(GRAD_STD).view(-1, BLOCK) * rows).view(-1).square_()
    s["primary"] = s["p"].to(torch.bfloat16)
    if case["states"] == "f32":
        s["m"], s["v"] = m, v
    else:
        s["m"], s["v"] = _encode_m(m.view(-1, BLOCK)), _encode_v(v.view(-1, BLOCK))
        s["m32"], s["v32"] = torch.empty_like(m), torch.empty_like(m)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    make = dict(rotary=_prepare_rotary, log_probs=_prepare_log_probs, adam=_prepare_adam)
    return dict(make[case["op"]](case, gen), case=case)


# --------------------------------------------------------------------------
# The plain forms
# --------------------------------------------------------------------------
def _plain_rotate(x, out, s, way):
    case = s["case"]
    n = case["rotated"]
    angle = (s["positions"].double()[:, None] * s["turns"] * (2 * math.pi))[:, None, None, :]
    cos = torch.cos(angle).float() * case["scale"]
    sin = torch.sin(angle).float() * (case["scale"] if way == "forward" else -case["scale"])
    first = (..., slice(0, n, 2)) if case["interleaved"] else (..., slice(0, n // 2))
    second = (..., slice(1, n, 2)) if case["interleaved"] else (..., slice(n // 2, n))
    a, b = x[first].float(), x[second].float()
    out[first] = (a * cos - b * sin).to(out.dtype)
    out[second] = (a * sin + b * cos).to(out.dtype)
    if out is not x and n < case["dim"]:
        out[..., n:] = x[..., n:]


def _plain_rotary(s):
    way = s["case"]["way"]
    if way != "backward":
        _plain_rotate(s["x"], s["out"], s, "forward")
        if s["k"] is not None:
            _plain_rotate(s["k"], s["k_out"], s, "forward")
    if way != "forward":
        x, k = (s["out"], s["k_out"]) if way == "both" else (s["x"], s["k"])
        _plain_rotate(x, s["out"], s, "backward")
        if k is not None:
            _plain_rotate(k, s["k_out"], s, "backward")
    return dict(x=s["out"], k=s["k_out"])


def _plain_log_probs(s):
    case, x, targets = s["case"], s["x"].float(), s["targets"]
    out = {}
    valid = targets >= 0
    at = targets.clamp(min=0)[:, None]
    if case["way"] == "backward":
        lse, entropies = s["lse"], s["entropies"]
    else:
        most = x.amax(1)
        e = torch.exp(x - most[:, None])
        total = e.sum(1)
        lse = most + torch.log(total)
        out["log_probs"] = torch.where(valid, x.gather(1, at)[:, 0] - lse, torch.zeros_like(lse))
        out["lse"] = lse
        if case["entropy"]:
            part = torch.where(e > 0, e * (x - most[:, None]), torch.zeros_like(e))
            entropies = torch.log(total) - part.sum(1) / total
            out["entropies"] = entropies
        if case["top"]:
            # one key for a logit and its place, so that the lower of equals is first
            bits = (x + 0.0).view(torch.int32)  # the zeros are one number
            order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
            place = torch.arange(case["vocab"], device=x.device)
            key = order * (1 << 32) + ((1 << 32) - 1 - place)
            best = torch.topk(key, case["top"], dim=1).indices
            out["top_ids"] = best.int()
            out["top_log_probs"] = x.gather(1, best) - lse[:, None]
    if case["way"] != "forward":
        logs = x - lse[:, None]
        p = torch.exp(logs)
        g = torch.where(valid, s["dlog_probs"], torch.zeros_like(lse))
        dx = p * -g[:, None]
        if case["entropy"]:
            inner = torch.where(p > 0, p * (logs + entropies[:, None]), torch.zeros_like(p))
            dx = dx - s["dentropies"][:, None] * inner
        dx.scatter_add_(1, at, g[:, None])
        out["dx"] = dx.to(s["dx"].dtype)
    return out


# Moments in 8 bits, blocks of 256 values.  The first moment: int8 codes of
# scale = max / 127, code = rint(m * (127 / max)); a block whose largest is below
# 2^-100 is held as zeros.  The second: its root r in uint8 codes c of scale =
# max / 255^2, r = c^2 scale, c the largest integer with (c - 1/2)^2 <= r (255^2 / max)
# and at least 1 where r is not 0.  Every quotient and product is rounded to 32 bits.
def _divided(a, b):
    """a / b in 64 bits, rounded to 32."""
    return (a / b).float()


def _encode_m(m):
    most = m.abs().amax(1, keepdim=True)
    held = most >= 2.0 ** -100
    inv = torch.where(held, _divided(127.0, most.double()), torch.zeros_like(most))
    scale = torch.where(held, _divided(most.double(), 127.0), torch.zeros_like(most))
    return torch.round(m * inv).to(torch.int8).view(-1), scale.view(-1)


def _encode_v(v):
    r = torch.sqrt(v.double()).float()
    most = r.amax(1, keepdim=True)
    inv = torch.where(most > 0, _divided(65025.0, most.double()), torch.zeros_like(most))
    code = torch.floor(torch.sqrt((r * inv).double()) + 0.5)
    code = torch.where(r > 0, code.clamp(min=1), code)
    return code.to(torch.uint8).view(-1), _divided(most.double(), 65025.0).view(-1)


def _decode_m(state):
    return state[0].view(-1, BLOCK).float() * state[1][:, None]


def _decode_root(state):
    return state[0].view(-1, BLOCK).float().square() * state[1][:, None]


def _f32(x):
    """A number as 32 bits hold it."""
    return float(torch.tensor(x, dtype=torch.float32))


def _plain_adam(s):
    case = s["case"]
    b1, b2, lr = _f32(BETA1), _f32(BETA2), _f32(LR)
    rest1, rest2 = _f32(1 - b1), _f32(1 - b2)
    step, correct2 = lr / (1 - b1 ** STEP), 1 / (1 - b2 ** STEP)
    p, g = s["p"].view(-1, BLOCK), s["g"].view(-1, BLOCK).float()
    small = case["states"] == "i8"
    m = _decode_m(s["m"]) if small else s["m"].view(-1, BLOCK)
    v = _decode_root(s["v"]).square() if small else s["v"].view(-1, BLOCK)
    # the moments decide codes: their sums in 64 bits, rounded once to 32
    m = (b1 * m.double() + (rest1 * g).double()).float()
    v = (b2 * v.double() + (rest2 * (g * g)).double()).float()
    fresh = p - (lr * s["decay"]) * p
    fresh = fresh - step * (m / (torch.sqrt(v * correct2) + _f32(EPS)))
    p.copy_(fresh)
    s["primary"].copy_(fresh.view(-1))
    out = dict(p=s["p"], primary=s["primary"])
    if not small:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        return dict(out, m=s["m"], v=s["v"])
    s["m"], s["v"] = _encode_m(m), _encode_v(v)
    return dict(out, m=_decode_m(s["m"]).view(-1), v=_decode_root(s["v"]).square().view(-1))


# --------------------------------------------------------------------------
# The framework's calls
# --------------------------------------------------------------------------
def _own_rotary(s):
    from paper_2407_01614_amd import zpp
    case = s["case"]
    how = dict(interleaved=case["interleaved"], scale=case["scale"])
    x, k = s["x"], s["k"]
    if case["way"] != "backward":
        zpp.rotary_forward(x, s["positions"], s["turns"], s["out"], k=k, k_out=s["k_out"], **how)
        x, k = s["out"], s["k_out"]
    if case["way"] != "forward":
        zpp.rotary_backward(x, s["positions"], s["turns"], s["out"], k=k, k_out=s["k_out"], **how)
    return dict(x=s["out"], k=s["k_out"])


def _workspace(s, nbytes):
    """The program's workspace: laid out on its first pass, then kept."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_log_probs(s):
    from paper_2407_01614_amd import zpp
    case, x, targets = s["case"], s["x"], s["targets"]
    entropies = s["entropies"] if case["entropy"] else None
    if case["way"] == "backward":
        zpp.log_probs_backward(x, targets, s["lse"], s["dlog_probs"], s["dx"],
                               entropies=entropies, dentropies=s.get("dentropies"))
        return dict(dx=s["dx"])
    out = dict(log_probs=s["log_probs"], lse=s["lse"])
    if case["entropy"]:
        out["entropies"] = entropies
    ws = _workspace(s, zpp.log_probs_workspace(case["rows"], case["vocab"], case["top"]))
    if case["way"] == "train":
        zpp.log_probs_train(x, targets, s["log_probs"], s["lse"], s["dlog_probs"], s["dx"], ws,
                            entropies=entropies, dentropies=s.get("dentropies"))
        return dict(out, dx=s["dx"])
    zpp.log_probs_forward(x, targets, s["log_probs"], s["lse"], ws, entropies=entropies,
                          top_ids=s.get("top_ids"), top_log_probs=s.get("top_log_probs"))
    if case["top"]:
        out.update(top_ids=s["top_ids"], top_log_probs=s["top_log_probs"])
    return out


def _own_adam(s):
    from paper_2407_01614_amd import zpp
    small = s["case"]["states"] == "i8"
    if "tensors" not in s:  # the program's list of tensors: written on its first pass, then kept
        def pieces(x, block=1):
            return [x[a // block:a // block + -(-n // block)]
                    for a, n in zip(s["starts"], s["lengths"])]

        m, v = ((list(zip(pieces(x[0]), pieces(x[1], BLOCK))) if small else pieces(x))
                for x in (s["m"], s["v"]))
        s["tensors"] = zpp.AdamTensors(pieces(s["p"]), m, v, pieces(s["g"]),
                                       pieces(s["primary"]), weight_decay=s["decays"])
    zpp.adam_tensors_step(s["tensors"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, step=STEP)
    out = dict(p=s["p"], primary=s["primary"])
    if not small:
        return dict(out, m=s["m"], v=s["v"])
    zpp.adam_state_load(s["m"], s["m32"])
    zpp.adam_state_load(s["v"], s["v32"])
    return dict(out, m=s["m32"], v=s["v32"])


def run(state):
    op = state["case"]["op"]
    if own:
        return dict(rotary=_own_rotary, log_probs=_own_log_probs, adam=_own_adam)[op](state)
    return dict(rotary=_plain_rotary, log_probs=_plain_log_probs, adam=_plain_adam)[op](state)


# --------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# --------------------------------------------------------------------------
def work(case):
    if case["op"] == "rotary":
        size = 4 if case["type"] == "f32" else 2
        heads = case["tokens"] * (case["heads"] + case["kv_heads"])
        # in place, features that do not turn are not touched
        touched = case["dim"] if case["layout"] == "separate" else case["rotated"]
        ways = 2 if case["way"] == "both" else 1
        return dict(bytes=2 * ways * heads * touched * size + 8 * case["tokens"],
                    flops=3 * ways * heads * case["rotated"])
    if case["op"] == "log_probs":
        size = 4 if case["type"] == "f32" else 2
        n = case["rows"] * case["vocab"]
        forward, backward = case["way"] != "backward", case["way"] != "forward"
        return dict(bytes=n * size * (2 if backward else 1) + case["rows"] * (24 + 8 * case["top"]),
                    flops=n * (4 * forward + 4 * backward) * (2 if case["entropy"] else 1))
    n = sum(_lengths(case))
    each = 8 + (4 if case["grad"] == "f32" else 2) + 2
    each += 16 if case["states"] == "f32" else 4 + 16 / BLOCK + 8
    return dict(bytes=n * each, flops=16 * n)


def _exact_entropy(x):
    logs = torch.log_softmax(x, 1)
    return -torch.where(torch.isinf(logs), torch.zeros_like(x), logs * torch.exp(logs)).sum(1)


def _exact_rotary(s):
    case = s["case"]
    n = case["rotated"]
    unit = torch.polar(torch.full((), case["scale"], dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None] * s["turns"] * (2 * math.pi))

    def turned(x, by):
        x = x.double()
        head = x[..., :n]
        if case["interleaved"]:
            pairs = head.unflatten(-1, (n // 2, 2))
        else:
            pairs = head.unflatten(-1, (2, n // 2)).transpose(-1, -2)
        z = torch.view_as_complex(pairs.contiguous()) * by[:, None, None, :]
        z = torch.view_as_real(z)
        head = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([head, x[..., n:]], -1)

    def passes(x):
        if x is None:
            return None
        if case["way"] != "backward":
            x = turned(x, unit).to(TYPES[case["type"]])
        return turned(x, unit.conj()).to(TYPES[case["type"]]) if case["way"] != "forward" else x

    if case["way"] == "both":
        return dict(x=passes(s["x"]), k=passes(s["k"]))
    by = unit if case["way"] == "forward" else unit.conj()
    return dict(x=turned(s["x"], by), k=None if s["k"] is None else turned(s["k"], by))


def _exact_log_probs(s):
    case, x, out = s["case"], s["x"].double(), {}
    valid = s["targets"] >= 0
    at = s["targets"].clamp(min=0)[:, None]
    if case["way"] == "backward":
        lse, entropies = s["lse"].double(), s["entropies"].double()
    else:
        lse = torch.logsumexp(x, 1)
        out.update(lse=lse, log_probs=(torch.gather(x, 1, at)[:, 0] - lse) * valid)
        if case["entropy"]:
            entropies = out["entropies"] = _exact_entropy(x)
        if case["top"]:
            best, ids = torch.sort(x, dim=1, descending=True, stable=True)
            out["top_ids"] = ids[:, :case["top"]].int()
            out["top_log_probs"] = best[:, :case["top"]] - lse[:, None]
    if case["way"] != "forward":
        g = s["dlog_probs"].double() * valid
        p = torch.exp(x - lse[:, None])
        dx = -g[:, None] * p
        if case["entropy"]:
            logs = (x - lse[:, None]).clamp(min=-1e4)  # a masked token's share is zero
            dx -= s["dentropies"].double()[:, None] * p * (logs + entropies[:, None])
        rows = torch.arange(case["rows"], device=x.device)
        dx[rows, at[:, 0]] += g
        out["dx"] = dx
    return out


def _exact_adam(s):
    case, out = s["case"], {}
    f = lambda t: t.float().double()  # noqa: E731  (rounded to 32 bits)
    b1, b2, lr, eps = (_f32(x) for x in (BETA1, BETA2, LR, EPS))
    g = s["g"].double()
    small = case["states"] == "i8"

    def spread(scale):
        return torch.repeat_interleave(scale.double(), BLOCK)

    if small:
        m = f(s["m"][0].double() * spread(s["m"][1]))
        v = f(f(s["v"][0].double() ** 2 * spread(s["v"][1])) ** 2)
    else:
        m, v = s["m"].double(), s["v"].double()
    m = b1 * m + f(_f32(1 - b1) * g)
    v = b2 * v + f(_f32(1 - b2) * f(g * g))
    p = s["p"].double() * (1 - lr * torch.repeat_interleave(s["decay"].double()[:, 0], BLOCK))
    p -= lr / (1 - b1 ** STEP) * m / (torch.sqrt(v / (1 - b2 ** STEP)) + eps)
    out.update(p=p, primary=p)
    if not small:
        return dict(out, m=m, v=v)
    del p, g
    # codes are decided by the moments as 32 bits hold them
    m, r = f(m).view(-1, BLOCK), f(torch.sqrt(f(v))).view(-1, BLOCK)
    top = m.abs().max(1).values[:, None]
    keep = (top >= 2.0 ** -100).double()
    top = top.clamp(min=2.0 ** -100)
    out["m"] = (torch.round(f(m * f(127 / top))) * f(top / 127) * keep).view(-1)
    del m
    top = r.max(1).values[:, None]
    some = top.clamp(min=2.0 ** -100)
    t = f(r * f(65025 / some))
    c = torch.sqrt(t).round()
    c = torch.where((c - 0.5) ** 2 > t, c - 1, c)
    c = torch.where((c + 0.5) ** 2 <= t, c + 1, c)
    c = torch.maximum(c, (r > 0).double())
    out["v"] = ((c * c * f(top / 65025)) ** 2).view(-1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return dict(rotary=_exact_rotary, log_probs=_exact_log_probs, adam=_exact_adam)[case["op"]](s)
