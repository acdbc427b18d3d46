"""The token operators (rotary positions, log probabilities with their gradient,
AdamW over many tensors) on the GPU against plain 64-bit forms, with the bounds of
tests/token_reference.py: types, layouts, odd sizes, strides, masks, empty calls,
gradients against differences, streams, captured calls, and the same bits on
every run."""
import itertools

import numpy as np
import pytest
import torch

import token_reference as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
INF = float("inf")


@pytest.fixture(scope="module")
def zpp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_01614_amd import zpp as mod
    return mod


def bits(t):
    return t.contiguous().view({2: torch.int16, 4: torch.int32, 1: torch.uint8}[t.element_size()])


def same(a, b):
    return torch.equal(bits(a), bits(b))


def assert_within(got, want, bound, dtype=F32):
    """|got - want| <= bound + the rounding of a result to its type."""
    got = got.double()
    off = (got - want).abs()
    allowed = bound + ref.out_step(dtype) * (want.abs() + bound)
    bad = ~(off <= allowed)
    assert not bool(bad.any()), "%d of %d, worst %g of its bound" % (
        int(bad.sum()), bad.numel(), float((off / allowed.clamp(min=1e-300)).max()))


# --------------------------------------------------------------------------
# Rotary positions
# --------------------------------------------------------------------------
# tokens, heads, key heads, dim, rotated: a token, odd ones, part of the head, one pair,
# pairs that no vector divides, wide heads, many heads, nothing that turns
ROTARY = [(1, 71, 1, 64, 64), (1, 1, 0, 2, 2), (333, 5, 5, 80, 20), (7, 3, 1, 10, 6),
          (130, 4, 2, 128, 128), (65, 2, 1, 320, 318), (3, 1, 1, 4112, 4096), (9, 150, 3, 64, 48),
          (2000, 4, 1, 32, 32), (1500, 2, 2, 26, 14), (5, 2, 1, 17, 0), (1100, 33, 1, 66, 62)]


def plan(zpp, tokens, rotated, far, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    positions = torch.randint(-far, far + 1, (tokens,), device="cuda", generator=gen)
    positions[0] = far
    return positions, zpp.rotary_turns(rotated, linear=2.0)


def heads(shape, seed, dtype, order="token"):
    """[tokens, groups, heads, dim], as stored, or with heads before tokens and a gap."""
    x = ref.numbers(shape, seed, dtype)
    if order == "head":
        big = torch.zeros(shape[1], shape[2], shape[0], shape[3] + 3, dtype=dtype, device="cuda")
        view = big.permute(2, 0, 1, 3)[..., 1:1 + shape[3]]
        view.copy_(x)
        return view
    return x


@TYPES
@pytest.mark.parametrize("near", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("size", ROTARY, ids=["%dx%d+%dx%d:%d" % s for s in ROTARY])
def test_rotary(zpp, size, near, dtype):
    tokens, h, kv, dim, rotated = size
    positions, turns = plan(zpp, tokens, rotated, 4000000 if tokens % 2 else 5000)
    for way, order, scale in ((zpp.rotary_forward, "token", 1.0), (zpp.rotary_backward, "head", 1.25)):
        x = heads((tokens, 1, h, dim), 3, dtype, order)
        k = heads((tokens, 1, kv, dim), 4, dtype) if kv else None
        out = torch.full_like(x, 7.0)
        k_out = None if k is None else heads((tokens, 1, kv, dim), 5, dtype, "head")
        how = dict(interleaved=near, scale=scale)
        way(x, positions, turns, out, k=k, k_out=k_out, **how)
        for a, b in ((x, out), (k, k_out)):
            if a is None:
                continue
            want, bound = ref.rotated(a, positions, turns, near, scale, way is zpp.rotary_backward)
            assert_within(b, want, bound, dtype)
            assert same(b[..., rotated:], a[..., rotated:])
        # in place, the same bits; every run the same bits
        again, k_again = x.clone(memory_format=torch.preserve_format), None if k is None else k.clone()
        way(again, positions, turns, again, k=k_again, k_out=k_again, **how)
        assert same(again, out) and (k is None or same(k_again, k_out))


def test_rotary_grouped_and_fused(zpp):
    """A key's head behind the query heads that share it, and query, key and value columns of
    one buffer, in place: the values stay as they are."""
    t, g, q, dim = 37, 3, 5, 64
    positions, turns = plan(zpp, t, 64, 8191)
    whole = ref.numbers((t, g, q + 2, dim), 1, BF16)
    for columns in ("one", "apart"):
        buffer = whole.clone()
        if columns == "one":
            x = buffer[:, :, :q + 1]
            zpp.rotary_forward(x, positions, turns, x)
        else:
            x, k = buffer[:, :, :q], buffer[:, :, q:q + 1]
            zpp.rotary_forward(x, positions, turns, x, k=k, k_out=k)
        want, bound = ref.rotated(whole[:, :, :q + 1], positions, turns, False, 1.0, False)
        assert_within(buffer[:, :, :q + 1], want, bound, BF16)
        assert same(buffer[:, :, q + 1:], whole[:, :, q + 1:])
    flat = whole.view(t, -1).clone()
    x, k = (flat[:, a * dim:b * dim].view(t, -1, dim) for a, b in ((0, 9), (9, 12)))
    zpp.rotary_forward(x, positions, turns, x, k=k, k_out=k)
    want, bound = ref.rotated(whole.view(t, 1, -1, dim)[:, :, :12], positions, turns, False, 1.0,
                              False)
    assert_within(flat.view(t, 1, -1, dim)[:, :, :12], want, bound, BF16)
    assert same(flat[:, 12 * dim:], whole.view(t, -1)[:, 12 * dim:])


def test_rotary_keeps_what_is_beside_it(zpp):
    positions, turns = plan(zpp, 9, 6, 100)
    for near in (False, True):
        big = torch.full((9, 3, 25), 5.0, dtype=F32, device="cuda")
        zpp.rotary_forward(ref.numbers((9, 2, 11), 1, F32), positions, turns, big[:, 1:, 7:18],
                           interleaved=near)
        assert bool((big[:, 0] == 5).all()) and bool((big[..., :7] == 5).all())
        assert bool((big[..., 18:] == 5).all())


def test_rotary_backward_is_the_transpose(zpp):
    """<forward(x), y> = <x, backward(y)>, and a unit vector's difference."""
    positions, turns = plan(zpp, 11, 12, 100)
    for near in (False, True):
        x, y = ref.numbers((11, 3, 16), 1, F32), ref.numbers((11, 3, 16), 2, F32)
        fx, by = torch.empty_like(x), torch.empty_like(y)
        how = dict(interleaved=near, scale=1.5)
        zpp.rotary_forward(x, positions, turns, fx, **how)
        zpp.rotary_backward(y, positions, turns, by, **how)
        a, b = (fx.double() * y.double()).sum(), (x.double() * by.double()).sum()
        # every element is off by at most 6 u of the pair's size times 1.5, both ways
        size = 1.5 * x.double().norm() * y.double().norm()
        assert abs(float(a - b)) <= 2 * 6 * 2 * ref.U * float(size)


def test_rotary_strange_numbers(zpp):
    positions, turns = plan(zpp, 4, 8, 50)
    x = ref.numbers((4, 2, 8), 1, BF16)
    x[1, 0, 2], x[2, 1, 5] = float("nan"), INF
    out = torch.empty_like(x)
    zpp.rotary_forward(x, positions, turns, out)
    bad = ~torch.isfinite(out)
    assert bool(bad[1, 0, 2]) and bool(bad[1, 0, 6]) and bool(bad[2, 1, 5]) and bool(bad[2, 1, 1])
    assert int(bad.sum()) == 4
    turns[1] = float("nan")
    zpp.rotary_forward(torch.ones_like(x), positions, turns, out)
    bad = torch.isnan(out)
    assert bool(bad[..., 1::4].all()) and int(bad.sum()) == 16


def test_rotary_empty(zpp):
    positions, turns = plan(zpp, 1, 8, 5)
    for shape in ((0, 3, 8), (4, 0, 8)):
        x = torch.empty(shape, dtype=BF16, device="cuda")
        p = torch.zeros(shape[0], dtype=torch.int64, device="cuda")
        ev = zpp.Event()
        zpp.rotary_forward(x, p, turns, torch.empty_like(x), done_after=ev)
        ev.synchronize()


def test_rotary_far_apart(zpp):
    """Offsets that pass 32 bits: tokens 2^31 elements apart."""
    far = (1 << 31) + 64
    big = torch.empty(far + 2 * 64, dtype=BF16, device="cuda")
    x = big.as_strided((2, 2, 64), (far, 64, 1))
    x.copy_(ref.numbers((2, 2, 64), 1, BF16))
    start = x.clone()
    positions, turns = plan(zpp, 2, 64, 77)
    zpp.rotary_forward(x, positions, turns, x)
    want, bound = ref.rotated(start[:, None], positions, turns, False, 1.0, False)
    assert_within(x[:, None], want, bound, BF16)


# --------------------------------------------------------------------------
# Log probabilities
# --------------------------------------------------------------------------
# rows, vocab, pad: one token, a chunk and less, odd ones, the lines between a row's ways
LOGITS = [(1, 1, 0), (3, 7, 1), (5, 64, 0), (70, 65, 3), (17, 1001, 7), (9, 1024, 0), (6, 1025, 0),
          (33, 2048, 8), (2, 2049, 1), (3, 4099, 0), (600, 4100, 0), (1, 8193, 0), (530, 8200, 3),
          (5, 16384, 0), (4, 16390, 131), (2, 32003, 5), (1, 65024, 0), (3, 65536, 1),
          (2, 65537, 0), (2, 131072, 0), (1, 262144, 0), (513, 2100, 0)]
EACH = pytest.mark.parametrize("rows,vocab,pad", LOGITS, ids=["%dx%d+%d" % s for s in LOGITS])


def logits(rows, vocab, pad, dtype, seed, masked=True):
    """Logits of every spread, a stretch masked, and targets of which some take no part."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((rows, vocab + pad), 3e4, dtype=dtype, device="cuda")[:, :vocab]
    spread = 10.0 ** torch.randint(-2, 2, (rows, 1), device="cuda", generator=gen)
    shift = 20 * torch.randn(rows, 1, device="cuda", generator=gen)
    x.copy_(spread * torch.randn(rows, vocab, device="cuda", generator=gen) + shift)
    keep = vocab - vocab // 3 if masked else vocab
    targets = torch.randint(keep, (rows,), device="cuda", generator=gen)
    x[torch.arange(rows, device="cuda"), targets] += 5 * torch.rand(rows, device="cuda",
                                                                    generator=gen).to(dtype)
    if masked:
        x[:, keep:] = -INF
    targets[1::4] = -100
    return x, targets


def workspace(zpp, rows, vocab, top=0):
    n = zpp.log_probs_workspace(rows, vocab, top)
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def outputs(rows, n=3):
    return [torch.full((rows,), 7.0, device="cuda") for _ in range(n)]


def check_forward(x, targets, lp, lse, h):
    vocab = x.shape[1]
    w_lse, ln, w_h, mean_d = ref.softmax_parts(x)
    at = targets.clamp(min=0)[:, None]
    w_lp = x.double().gather(1, at)[:, 0] - w_lse
    b_lse, b_lp, b_h = ref.forward_bounds(vocab, w_lse, ln, w_h, mean_d, w_lp)
    none = targets < 0
    assert bool((lp[none] == 0).all())
    assert_within(lp[~none], w_lp[~none], b_lp[~none])
    assert_within(lse, w_lse, b_lse)
    if h is not None:
        assert_within(h, w_h, b_h)


@TYPES
@EACH
def test_log_probs_forward(zpp, rows, vocab, pad, dtype):
    x, targets = logits(rows, vocab, pad, dtype, rows + vocab)
    ws = workspace(zpp, rows, vocab)
    lp, lse, h = outputs(rows)
    zpp.log_probs_forward(x, targets, lp, lse, ws, entropies=h)
    check_forward(x, targets, lp, lse, h)
    lp2, lse2, _ = outputs(rows)
    zpp.log_probs_forward(x, targets, lp2, lse2, ws)
    check_forward(x, targets, lp2, lse2, None)
    lp3, = outputs(rows, 1)
    zpp.log_probs_forward(x, targets, lp3, None, ws)
    assert same(lp3, lp2)


@TYPES
@EACH
def test_log_probs_backward_and_train(zpp, rows, vocab, pad, dtype):
    x, targets = logits(rows, vocab, pad, dtype, rows + vocab)
    g, dh = ref.numbers((rows,), 5, F32), ref.numbers((rows,), 6, F32, 0.1)
    w_lse, ln, w_h, mean_d = ref.softmax_parts(x)
    lse, h = w_lse.float(), w_h.float()
    rel = ref.sum_bound(vocab, mean_d) + 2 * ref.U * (ln.abs() + 1)
    ws = workspace(zpp, rows, vocab)
    for entropy in (False, True):
        more = dict(entropies=h, dentropies=dh) if entropy else {}
        parts = (dh, h.double()) if entropy else (None, None)
        dx = torch.full((rows, vocab + 5), 9.0, dtype=dtype, device="cuda")
        zpp.log_probs_backward(x, targets, lse, g, dx[:, :vocab], **more)
        want, bound = ref.gradient(x, targets, lse.double(), g, *parts)
        assert_within(dx[:, :vocab], want, bound, dtype)
        assert bool((dx[:, vocab:] == 9).all())
        # in place
        y = x.clone()
        zpp.log_probs_backward(y, targets, lse, g, y, **more)
        assert same(y, dx[:, :vocab])
        # both passes in one
        dx.fill_(9.0)
        lp, lse2, h2 = outputs(rows)
        more = dict(entropies=h2, dentropies=dh) if entropy else {}
        zpp.log_probs_train(x, targets, lp, lse2, g, dx[:, :vocab], ws, **more)
        check_forward(x, targets, lp, lse2, h2 if entropy else None)
        parts = (dh, w_h) if entropy else (None, None)
        want, bound = ref.gradient(x, targets, w_lse, g, *parts, rel_s=rel)
        assert_within(dx[:, :vocab], want, bound, dtype)
        assert bool((dx[:, vocab:] == 9).all())
        y, first = x.clone(), (lp.clone(), lse2.clone())
        zpp.log_probs_train(y, targets, lp, lse2, g, y, ws, **more)
        assert same(y, dx[:, :vocab]) and same(lp, first[0]) and same(lse2, first[1])


def test_log_probs_gradient_against_differences(zpp):
    """The loss sum(g lp + h entropy) by differences of its 64-bit form at the kernel's inputs."""
    rows, vocab = 4, 37
    x, targets = logits(rows, vocab, 0, F32, 3, masked=False)
    x.clamp_(-5, 5)
    g, dh = ref.numbers((rows,), 5, F32), ref.numbers((rows,), 6, F32)
    dx, (lp, lse, h) = torch.empty_like(x), outputs(rows)
    zpp.log_probs_train(x, targets, lp, lse, g, dx, None, entropies=h, dentropies=dh)

    def loss(x):
        logs = torch.log_softmax(x, 1)
        at = logs.gather(1, targets.clamp(min=0)[:, None])[:, 0] * (targets >= 0)
        return g.double() * at - dh.double() * (logs.exp() * logs).sum(1)

    step = 2.0 ** -14
    for j in range(vocab):
        up, down = x.double().clone(), x.double().clone()
        up[:, j] += step
        down[:, j] -= step
        diff = (loss(up) - loss(down)) / (2 * step)
        # third derivatives of these sums are below 64 (|g| + |dh|): step^2 / 6 of that; and
        # 64 u of the terms for the kernel
        size = g.double().abs() + 16 * dh.double().abs()
        assert bool(((dx[:, j].double() - diff).abs() <= size * (64 * step * step + 64 * ref.U)).all())


TOPS = [(1, 1, 1), (3, 7, 7), (2, 16, 16), (5, 64, 64), (3, 65, 64), (70, 300, 5), (1, 2048, 20),
        (2, 2049, 20), (77, 32003, 5), (1, 65024, 20), (4, 65024, 64), (300, 8200, 32),
        (2, 262144, 32), (1, 524288, 64), (130, 20011, 1), (1030, 2100, 3)]


@TYPES
@pytest.mark.parametrize("rows,vocab,top", TOPS, ids=["%dx%d:%d" % s for s in TOPS])
@pytest.mark.parametrize("kind", ["spread", "equal", "rising", "zeros", "few"])
def test_log_probs_top(zpp, rows, vocab, top, kind, dtype):
    x, targets = logits(rows, vocab, 3, dtype, rows + vocab)
    at = torch.arange(vocab, device="cuda")
    if kind == "equal":
        x[:] = 1.5
    elif kind == "rising":  # the largest lie side by side, at 2048 apart, or in one half
        x[:] = (at // 16).to(dtype)
        x[1::3] = (at % 2048).to(dtype) / 8
        x[2::3] = -at.to(dtype)
    elif kind == "zeros":   # both zeros are one number
        x[:] = torch.where(at % 3 == 0, -0.0, 0.0).to(dtype)
        x[:, vocab // 2] = 2.0
    elif kind == "few":     # fewer unmasked than asked for
        x[:] = -INF
        x[:, vocab // 2] = 1.0
        targets[:] = vocab // 2
    ids = torch.full((rows, top), -1, dtype=torch.int32, device="cuda")
    tlp, (lp, lse, h) = torch.full((rows, top), 7.0, device="cuda"), outputs(rows)
    ws = workspace(zpp, rows, vocab, top)
    zpp.log_probs_forward(x, targets, lp, lse, ws, entropies=h, top_ids=ids, top_log_probs=tlp)
    want = ref.top_ids(x, top)
    assert torch.equal(ids.long(), want)
    check_forward(x, targets, lp, lse, h)
    w_lse, ln, _, mean_d = ref.softmax_parts(x)
    w = x.double().gather(1, want) - w_lse[:, None]
    _, bound, _ = ref.forward_bounds(vocab, w_lse[:, None], ln[:, None], ln[:, None],
                                     mean_d[:, None], torch.where(torch.isinf(w), 0, w))
    inf = torch.isinf(w)
    assert torch.equal(torch.isinf(tlp), inf) and bool((tlp[inf] < 0).all())
    assert_within(tlp[~inf], w[~inf], bound.expand_as(w)[~inf])


@TYPES
@pytest.mark.parametrize("vocab", [5, 700, 5000, 30000, 66000])
def test_log_probs_strange_rows(zpp, vocab, dtype):
    """A row masked throughout by -Inf, by the type's lowest, NaN, +Inf, a masked target, a target past
    the vocabulary, the largest numbers, and a plain row beside them."""
    rows, top = 8, min(vocab, 4)
    x, targets = logits(rows, vocab, 1, dtype, vocab, masked=False)
    targets.fill_(2)
    lowest = torch.finfo(dtype).min
    x[0] = -INF
    x[1] = lowest
    x[2, vocab - 1] = float("nan")
    x[3, 1] = INF
    x[4, 2] = -INF
    targets[5] = vocab
    x[6] = -lowest
    x[6, 3:] = lowest
    g, dh = torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda")
    ws, ws_top = workspace(zpp, rows, vocab), workspace(zpp, rows, vocab, top)
    runs = []
    for way in ("forward", "top", "train"):
        lp, lse, h = outputs(rows)
        if way == "train":
            dx = torch.full_like(x, 3.0)
            zpp.log_probs_train(x, targets, lp, lse, g, dx, ws, entropies=h, dentropies=dh)
            runs.append(dx)
            dx = torch.full_like(x, 3.0)
            zpp.log_probs_backward(x, targets, lse, g, dx, entropies=h, dentropies=dh)
            runs.append(dx)
        elif way == "top":
            ids = torch.full((rows, top), -1, dtype=torch.int32, device="cuda")
            tlp = torch.zeros(rows, top, device="cuda")
            zpp.log_probs_forward(x, targets, lp, lse, ws_top, entropies=h, top_ids=ids,
                                  top_log_probs=tlp)
            assert bool(((ids >= 0) & (ids < vocab)).all())
            assert bool((tlp[0] == -INF).all()) and bool(torch.isnan(tlp[2:4]).all())
        else:
            zpp.log_probs_forward(x, targets, lp, lse, ws, entropies=h)
        assert float(lp[0]) == float(lse[0]) == -INF and float(h[0]) == 0
        n = np.log(vocab)
        assert abs(float(lp[1]) + n) < 1e-4 and abs(float(h[1]) - n) < 1e-4
        assert float(lse[1]) == lowest
        assert bool(torch.isnan(torch.stack([lp[2:4], lse[2:4], h[2:4]])).all())
        assert float(lp[4]) == -INF and np.isfinite(float(lse[4]))
        assert np.isnan(float(lp[5])) and np.isfinite(float(lse[5]))
        assert abs(float(lp[6]) + np.log(3)) < 1e-6 and abs(float(h[6]) - np.log(3)) < 1e-6
        w_lse, ln, w_h, mean_d = ref.softmax_parts(x[7:])
        w_lp = x[7:].double()[:, 2] - w_lse
        b = ref.forward_bounds(vocab, w_lse, ln, w_h, mean_d, w_lp)
        assert_within(lse[7:], w_lse, b[0])
        assert_within(lp[7:], w_lp, b[1])
    for dx in runs:
        assert bool((dx[0] == 0).all())
        assert bool(torch.isnan(dx[2]).all()) and bool(torch.isnan(dx[5]).all())
        assert bool(torch.isfinite(dx[4]).all()) and float(dx[4, 2]) == 1.0
        assert bool((dx[6, 3:] == 0).all())


def test_log_probs_empty(zpp):
    ev = zpp.Event()
    x, t = torch.empty(0, 40, dtype=BF16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    lp, lse, h = outputs(0)
    zpp.log_probs_forward(x, t, lp, lse, None, done_after=ev)
    zpp.log_probs_backward(x, t, lse, lp, torch.empty_like(x))
    zpp.log_probs_train(x, t, lp, lse, h, torch.empty_like(x), None)
    ev.synchronize()


def test_log_probs_far_apart(zpp):
    """Rows 2^31 elements apart."""
    far, vocab = (1 << 31) + 8, 5000
    big = torch.empty(2 * far + vocab, dtype=BF16, device="cuda")
    x = big.as_strided((3, vocab), (far, 1))
    y, targets = logits(3, vocab, 0, BF16, 4)
    x.copy_(y)
    lp, lse, h = outputs(3)
    zpp.log_probs_forward(x, targets, lp, lse, workspace(zpp, 3, vocab), entropies=h)
    check_forward(y, targets, lp, lse, h)
    zpp.log_probs_train(x, targets, lp, lse, torch.ones(3, device="cuda"), x, workspace(zpp, 3, vocab))
    dy = torch.empty_like(y)
    zpp.log_probs_train(y, targets, lp, lse, torch.ones(3, device="cuda"), dy,
                        workspace(zpp, 3, vocab))
    assert same(x, dy)


@pytest.mark.parametrize("rows,vocab", [(5000, 40), (70000, 16), (3000, 3000)])
def test_log_probs_many_rows(zpp, rows, vocab):
    x, targets = logits(rows, vocab, 0, F32, 9)
    lp, lse, h = outputs(rows)
    ws = workspace(zpp, rows, vocab)
    zpp.log_probs_forward(x, targets, lp, lse, ws, entropies=h)
    check_forward(x, targets, lp, lse, h)
    g, dx = ref.numbers((rows,), 5, F32), torch.empty_like(x)
    zpp.log_probs_train(x, targets, lp, lse, g, dx, ws)
    check_forward(x, targets, lp, lse, None)
    w_lse, ln, _, mean_d = ref.softmax_parts(x)
    want, bound = ref.gradient(x, targets, w_lse, g,
                               rel_s=ref.sum_bound(vocab, mean_d) + 2 * ref.U * (ln.abs() + 1))
    assert_within(dx, want, bound)


# --------------------------------------------------------------------------
# AdamW over many tensors
# --------------------------------------------------------------------------
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


def tensors_of(lengths, seed, grad=F32, offset=0):
    """p, m, v, g, primary of each length, `offset` elements into an allocation."""
    found = []
    for i, n in enumerate(lengths):
        def one(std, dtype=F32, k=0):
            t = torch.empty(n + offset, dtype=dtype, device="cuda")[offset:]
            t.copy_(ref.numbers((n,), 31 * seed + 7 * i + k, F32, std))
            return t
        found.append((one(0.02), one(1e-3, k=1), one(1e-3, k=2).square_(), one(1e-2, grad, 3),
                      one(0, BF16)))
    return [list(x) for x in zip(*found)]


def stepped(zpp, p, m, v, g, wd, step, adamw):
    """The one-tensor step on copies, and its bf16 copy."""
    p, m, v = (t.clone() for t in (p, m, v))
    out = torch.empty(p.numel(), dtype=BF16, device="cuda")
    zpp.adam_partition_step(p, m, v, g.float().contiguous(), out, step=step, weight_decay=wd,
                            adamw=adamw, **HP)
    return p, m, v, out


LENGTHS = [[1], [255, 256, 257], [4096] * 65, list(range(1, 200)), [3, 0, 5, 0], [100000, 7, 513],
           [1] * 4097, [777] * 64 + [300]]
LISTS = pytest.mark.parametrize("lengths", LENGTHS, ids=["one", "block", "norms", "rising", "holes",
                                                         "large", "4097", "65"])


@LISTS
@pytest.mark.parametrize("grad", [F32, BF16], ids=["gf32", "gbf16"])
@pytest.mark.parametrize("adamw", [True, False], ids=["adamw", "l2"])
def test_adam_tensors_f32(zpp, lengths, grad, adamw):
    p, m, v, g, out = tensors_of(lengths, 1, grad, offset=1)
    decays = [0.1 * (i % 3) for i in range(len(p))]
    some = range(len(p)) if len(p) < 100 else [0, 1, 63, 64, 65, 127, 128, len(p) - 1]
    want = {i: stepped(zpp, p[i], m[i], v[i], g[i], decays[i], 3, adamw) for i in some}
    kept = [t.clone() for t in g]
    lists = zpp.AdamTensors(p, m, v, g, out, weight_decay=decays)
    zpp.adam_tensors_step(lists, step=3, adamw=adamw, **HP)
    for i in some:
        for a, b in zip((p[i], m[i], v[i], out[i]), want[i]):
            assert same(a, b), i
    assert all(same(a, b) for a, b in zip(g, kept))


def state8(x, moment):
    codes, scales = ref.encode_state(x.cpu().numpy(), moment)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()


def values8(state, moment):
    return torch.from_numpy(ref.decode_state(state[0].cpu().numpy(), state[1].cpu().numpy(),
                                             moment)).cuda()


@LISTS
@pytest.mark.parametrize("grad", [F32, BF16], ids=["gf32", "gbf16"])
def test_adam_tensors_i8(zpp, lengths, grad):
    """Codes, scales and weights, bit for bit: the one-tensor step on the values that the codes
    stand for, its moments encoded by the format's numpy form."""
    p, m, v, g, out = tensors_of(lengths, 2, grad, offset=1)
    m8, v8 = [state8(t, 1) for t in m], [state8(t, 2) for t in v]
    lists = zpp.AdamTensors(p, m8, v8, g, [None if i % 4 == 3 else t for i, t in enumerate(out)],
                            weight_decay=0.1)
    some = range(len(p)) if len(p) < 100 else [0, 1, 63, 64, 65, 127, 128, len(p) - 1]
    for step in (1, 2):
        want = {i: stepped(zpp, p[i], values8(m8[i], 1), values8(v8[i], 2), g[i], 0.1, step, True)
                for i in some}
        zpp.adam_tensors_step(lists, step=step, **HP)
        for i in some:
            assert same(p[i], want[i][0])
            if i % 4 == 3:
                assert bool((out[i] == 0).all())
            else:
                assert same(out[i], want[i][3])
            for state, x, moment in ((m8[i], want[i][1], 1), (v8[i], want[i][2], 2)):
                codes, scales = state8(x, moment)
                assert torch.equal(state[0], codes) and same(state[1], scales), (i, moment)


def hard_moments(n, seed, moment):
    """Blocks of every magnitude, with values on and beside the codes' borders, zeros, Inf, NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(n) * np.repeat(2.0 ** rng.integers(-80, 60, -(-n // 256)), 256)[:n]
    if moment == 1:
        x[::7] = rng.integers(-254, 255, x[::7].shape) / 2.0
        x[256 * 3:256 * 4] = rng.standard_normal(256)[:len(x[256 * 3:256 * 4])] * 2.0 ** -103
    else:
        c = rng.integers(0, 256, x[::5].shape)
        x[::5] = (c + 0.5) ** 4                       # roots on a border, where max is 255^2
        x[::256] = 65025.0 ** 2
        x = np.abs(x)
    x[256 * 5:256 * 6] = 0
    x[min(n - 1, 256 * 7)] = np.inf
    x[min(n - 1, 256 * 8 + 3)] = np.nan
    return torch.from_numpy(x.astype(np.float32)).cuda()


@pytest.mark.parametrize("n", [1, 3, 255, 256, 257, 5000, 100003])
@pytest.mark.parametrize("moment", [1, 2])
def test_adam_state_save_and_load(zpp, n, moment):
    x = hard_moments(n, n, moment)
    codes = torch.full((n + 2,), 99, dtype=torch.int8 if moment == 1 else torch.uint8, device="cuda")
    scales = torch.full((-(-n // 256) + 2,), 99.0, device="cuda")
    state = (codes[1:-1], scales[1:-1])
    zpp.adam_state_save(x, state)
    want = state8(x, moment)
    assert torch.equal(state[0], want[0])
    assert same(state[1].nan_to_num(nan=-1), want[1].nan_to_num(nan=-1))
    assert int(codes[0]) == int(codes[-1]) == 99 and float(scales[0]) == float(scales[-1]) == 99
    out = torch.full((n + 1,), 5.0, device="cuda")
    zpp.adam_state_load(state, out[:n])
    assert same(out[:n].nan_to_num(nan=-1), values8(want, moment).nan_to_num(nan=-1))
    assert float(out[n]) == 5.0


def test_adam_state_is_what_a_second_save_keeps(zpp):
    """What is read back is saved as the same values again: first moments exactly, a block's
    largest being its code 127; second ones too."""
    for moment in (1, 2):
        x = ref.numbers((4096,), 3, F32)
        x = x if moment == 1 else x.square()
        state = zpp.empty_adam_state(4096, moment)
        out = torch.empty_like(x)
        zpp.adam_state_load(state, out)
        assert bool((out == 0).all())
        zpp.adam_state_save(x, state)
        zpp.adam_state_load(state, out)
        top = x.view(-1, 256).abs().amax(1, keepdim=True).double()
        # half a step of a code: of 127 steps for the first; for the second the root's is
        # between (c -+ 1/2)^2, at most (c + 1/4) (max / 255^2) off; roundings 4 u
        if moment == 1:
            off = (out.double() - x.double()).view(-1, 256).abs()
            assert bool((off <= top / 254 * (1 + 8 * ref.U)).all())
        else:
            r, w = out.double().sqrt().view(-1, 256), x.double().sqrt().view(-1, 256)
            c = (w / top.sqrt() * 65025).sqrt()
            # codes kept to 1 stand for roots from 0 on
            room = torch.maximum(c + 0.25, torch.ones_like(c)) * (top.sqrt() / 65025)
            assert bool(((r - w).abs() <= room * (1 + 1e-4) + 8 * ref.U * w).all())


def test_adam_tensors_bad_block(zpp):
    """An Inf gradient reaches its element's weight and its block's moments, no other block's."""
    n = 1000
    (p,), (m,), (v,), (g,), (out,) = tensors_of([n], 4)
    g[300] = INF
    m8, v8 = state8(m, 1), state8(v, 2)
    zpp.adam_tensors_step(zpp.AdamTensors([p], [m8], [v8], [g], [out]), step=1, **HP)
    bad = ~torch.isfinite(p)
    assert bool(bad[300]) and int(bad.sum()) == 1
    for s in (m8[1], v8[1]):
        assert torch.isnan(s).tolist() == [False, True, False, False]
    assert bool((m8[0][256:512] == 0).all())


def test_adam_tensors_none(zpp):
    ev = zpp.Event()
    for lists in (zpp.AdamTensors([], [], [], []),
                  zpp.AdamTensors(*[[torch.empty(0, device="cuda")]] * 4)):
        zpp.adam_tensors_step(lists, step=1, done_after=ev, **HP)
        ev.synchronize()


# --------------------------------------------------------------------------
# Streams, captured calls
# --------------------------------------------------------------------------
def test_streams_and_events(zpp):
    """Work on a stream that waits for another's event, and is waited for."""
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    rows, vocab = 300, 30000
    x, targets = logits(rows, vocab, 0, BF16, 1)
    y = torch.zeros_like(x)
    (lp, lse, h), dx = outputs(rows), torch.empty_like(x)
    ids = torch.empty(rows, 5, dtype=torch.int32, device="cuda")
    tlp = torch.empty(rows, 5, device="cuda")
    ws = workspace(zpp, rows, vocab, 5)
    torch.cuda.synchronize()
    filled, done = zpp.Event(), zpp.Event()
    with torch.cuda.stream(a):
        torch.cuda._sleep(20000000)
        y.copy_(x)
        filled.record(a)
    zpp.log_probs_forward(y, targets, lp, lse, ws, entropies=h, top_ids=ids, top_log_probs=tlp,
                          stream=b, wait_before=filled, done_after=done)
    done.synchronize()
    check_forward(x, targets, lp, lse, h)
    assert torch.equal(ids.long(), ref.top_ids(x, 5))
    torch.cuda.synchronize()


def test_captured_step(zpp):
    """Rotary, both ways, the loss with its gradient and both kinds of step, captured and replayed
    with eager work between: the same bits as the eager calls.  Two graphs share a workspace
    one after the other."""
    t, h, dim, vocab = 40, 6, 64, 9000
    positions, turns = plan(zpp, t, dim, 5000)
    x0, (l0, targets) = ref.numbers((t, h, dim), 1, BF16), logits(3, vocab, 0, BF16, 2)
    g = ref.numbers((3,), 5, F32)
    start = tensors_of([300, 4096, 77], 6)
    ws, ws_top = workspace(zpp, 3, vocab), workspace(zpp, 3, vocab, 20)

    def state():
        p, m, v, gr, out = [[t.clone() for t in x] for x in start]
        s = dict(x=x0.clone(), l=l0.clone(), dx=torch.empty_like(l0), o=outputs(3), p=p, out=out,
                 ids=torch.zeros(3, 20, dtype=torch.int32, device="cuda"),
                 tlp=torch.zeros(3, 20, device="cuda"), q=[t.clone() for t in p])
        s["m8"], s["v8"] = [state8(t, 1) for t in m], [state8(t, 2) for t in v]
        s["f32"] = zpp.AdamTensors(p, m, v, gr, out, weight_decay=0.1)
        s["i8"] = zpp.AdamTensors(s["q"], s["m8"], s["v8"], gr, weight_decay=0.1)
        return s

    def work(s, stream=None):
        lp, lse, ent = s["o"]
        zpp.rotary_forward(s["x"], positions, turns, s["x"], stream=stream)
        zpp.rotary_backward(s["x"], positions, turns, s["x"], interleaved=True, stream=stream)
        zpp.log_probs_train(s["l"], targets, lp, lse, g, s["dx"], ws, stream=stream)
        zpp.log_probs_forward(s["l"], targets, lp, lse, ws_top, entropies=ent, top_ids=s["ids"],
                              top_log_probs=s["tlp"], stream=stream)
        zpp.adam_tensors_step(s["f32"], step=2, stream=stream, **HP)
        zpp.adam_tensors_step(s["i8"], step=2, stream=stream, **HP)

    def results(s):
        return [s["x"], s["dx"], *s["o"], s["ids"], s["tlp"], *s["p"], *s["q"], *s["out"],
                *itertools.chain(*s["m8"]), *itertools.chain(*s["v8"])]

    eager, two = state(), [state(), state()]
    graphs = []
    for s in two:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            work(s)
        graphs.append(graph)
    for _ in range(3):
        work(eager)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for s in two:
            assert all(same(a, b) for a, b in zip(results(eager), results(s)))


def test_side_stream_of_torch(zpp):
    """The current torch stream is where a call without one goes."""
    s = torch.cuda.Stream()
    x = ref.numbers((64, 8, 64), 1, BF16)
    positions, turns = plan(zpp, 64, 64, 999)
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(10000000)
        y = x.clone()
        zpp.rotary_forward(y, positions, turns, out)
    s.synchronize()
    want, bound = ref.rotated(x[:, None], positions, turns, False, 1.0, False)
    assert_within(out[:, None], want, bound, BF16)
