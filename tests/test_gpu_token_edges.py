"""The token operators where their kernels change over: rows that fill half or all of a
workgroup's registers, rows that begin inside a word, lists of the best tokens that
overflow, moments next to the codes' borders and below the normal numbers, heads whose
pairs no vector divides; and a training step that uses them together.  The bounds are those
of tests/token_reference.py."""
import numpy as np
import pytest
import torch

import token_reference as ref
from test_gpu_token_operators import (BF16, F32, HP, INF, TYPES, assert_within, check_forward,
                                      logits, outputs, plan, same, state8, values8, workspace)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zpp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_01614_amd import zpp as mod
    return mod


# --------------------------------------------------------------------------
# Log probabilities
# --------------------------------------------------------------------------
# (more rows than CUs: workgroups of 512 and 1024 lanes with 32 and 64 registers of a row,
# and in fp32 the two passes)
LONG = [(300, 8191), (300, 16385), (300, 20000), (260, 32769), (260, 40001), (260, 65537),
        (257, 70000)]


@TYPES
@pytest.mark.parametrize("rows,vocab", LONG, ids=["%dx%d" % s for s in LONG])
@pytest.mark.parametrize("pad", [0, 1])
def test_rows_in_registers(zpp, rows, vocab, pad, dtype):
    x, targets = logits(rows, vocab, pad, dtype, rows + vocab)
    g, dh = ref.numbers((rows,), 5, F32), ref.numbers((rows,), 6, F32, 0.1)
    w_lse, ln, w_h, mean_d = ref.softmax_parts(x)
    rel = ref.sum_bound(vocab, mean_d) + 2 * ref.U * (ln.abs() + 1)
    lp, lse, h = outputs(rows)
    dx = torch.full((rows, vocab + pad), 9.0, dtype=dtype, device="cuda")
    ws = workspace(zpp, rows, vocab)
    zpp.log_probs_train(x, targets, lp, lse, g, dx[:, :vocab], ws, entropies=h, dentropies=dh)
    check_forward(x, targets, lp, lse, h)
    want, bound = ref.gradient(x, targets, w_lse, g, dh, w_h, rel_s=rel)
    assert_within(dx[:, :vocab], want, bound, dtype)
    assert bool((dx[:, vocab:] == 9).all())
    first = lp.clone(), lse.clone(), h.clone()
    zpp.log_probs_train(x, targets, lp, lse, g, x, ws, entropies=h, dentropies=dh)
    assert same(x, dx[:, :vocab])
    assert all(same(a, b) for a, b in zip((lp, lse, h), first))


@TYPES
@pytest.mark.parametrize("rows,vocab,pad", [(1, 40000, 0), (100, 65024, 0), (150, 100003, 1),
                                            (257, 131073, 0)])
def test_rows_of_one_workgroup(zpp, rows, vocab, pad, dtype):
    """Few rows, too long for one batch, whole in a workgroup of 1024."""
    x, targets = logits(rows, vocab, pad, dtype, rows)
    lp, lse, h = outputs(rows)
    ws = workspace(zpp, rows, vocab)
    zpp.log_probs_forward(x, targets, lp, lse, ws, entropies=h)
    check_forward(x, targets, lp, lse, h)
    lp2, lse2, _ = outputs(rows)
    zpp.log_probs_forward(x, targets, lp2, lse2, ws)
    check_forward(x, targets, lp2, lse2, None)


@pytest.mark.parametrize("vocab", [9, 130, 2047, 8200, 33000])
@pytest.mark.parametrize("offset", [1, 2, 7])
def test_rows_that_begin_inside_a_word(zpp, vocab, offset):
    """A slice of wider rows from any column on: the bits of an array of its own."""
    rows = 9
    whole, targets = logits(rows, vocab, 0, BF16, vocab)
    big = torch.full((rows, vocab + 13), float("nan"), dtype=BF16, device="cuda")
    x = big[:, offset:offset + vocab]
    x.copy_(whole)
    g, ws = ref.numbers((rows,), 5, F32), workspace(zpp, rows, vocab)
    top = min(vocab, 5)
    ws_top = workspace(zpp, rows, vocab, top)
    found = []
    for a in (whole, x):
        lp, lse, h = outputs(rows)
        ids = torch.empty(rows, top, dtype=torch.int32, device="cuda")
        tlp = torch.empty(rows, top, device="cuda")
        lp2, lse2, _ = outputs(rows)
        dx = torch.full_like(big, 3.0)
        zpp.log_probs_forward(a, targets, lp, lse, ws, entropies=h)
        zpp.log_probs_forward(a, targets, lp2, lse2, ws_top, top_ids=ids, top_log_probs=tlp)
        zpp.log_probs_train(a, targets, lp2, lse2, g, dx[:, offset:offset + vocab], ws)
        assert bool((dx[:, :offset] == 3).all()) and bool((dx[:, offset + vocab:] == 3).all())
        found.append((lp, lse, h, ids, tlp, dx))
    assert all(same(a, b) for a, b in zip(*found))
    check_forward(x, targets, *found[1][:3])


@TYPES
@pytest.mark.parametrize("rows,vocab,top", [(2, 1000, 64), (2, 2048, 64), (3, 8192, 64),
                                            (520, 30000, 64), (1100, 2048, 64), (2, 70000, 64),
                                            (5, 33000, 64), (200, 100003, 7), (300, 9000, 9),
                                            (2, 524288, 1), (600, 20000, 2)])
def test_lists_that_overflow(zpp, rows, vocab, top, dtype):
    """Rows that rise, equal rows, rows of two values, a row masked but for a few, in turn."""
    at = torch.arange(vocab, device="cuda")
    x = torch.empty(rows, vocab, dtype=dtype, device="cuda")
    kinds = [at // 512, torch.zeros_like(at), at % 2, (at * 7919) % 251, -at // 8]
    for i in range(rows):
        x[i] = kinds[i % len(kinds)].to(dtype)
    x[rows - 1] = -INF
    few = torch.tensor([vocab // 2, vocab - 1, 3], device="cuda")
    x[rows - 1, few] = torch.tensor([1.0, 2.0, 1.0], dtype=dtype, device="cuda")
    targets = torch.zeros(rows, dtype=torch.int64, device="cuda")
    targets[rows - 1] = 3
    ids = torch.full((rows, top), -1, dtype=torch.int32, device="cuda")
    tlp, (lp, lse, h) = torch.full((rows, top), 7.0, device="cuda"), outputs(rows)
    zpp.log_probs_forward(x, targets, lp, lse, workspace(zpp, rows, vocab, top), entropies=h,
                          top_ids=ids, top_log_probs=tlp)
    assert torch.equal(ids.long(), ref.top_ids(x, top))
    want = x.double().gather(1, ids.long()) - ref.softmax_parts(x)[0][:, None]
    assert torch.equal(torch.isinf(tlp), torch.isinf(want))
    check_forward(x, targets, lp, lse, h)


@pytest.mark.parametrize("vocab", [9, 100, 1500, 9000, 70000])
@pytest.mark.parametrize("shift", [1e3, -3e4, 3e5, 1e6, -1e7, 1e8])
def test_large_logits(zpp, vocab, shift):
    """Logits far from 0 in fp32: log probabilities and gradients depend on their differences,
    which are exact."""
    rows = 5
    ulp = float(np.spacing(np.float32(abs(shift))))
    steps = torch.randn(rows, vocab, device="cuda",
                        generator=torch.Generator(device="cuda").manual_seed(vocab))
    x = (shift + (3 * steps / ulp).round().double() * ulp).float()
    targets = torch.arange(rows, device="cuda")
    g, dh = ref.numbers((rows,), 5, F32), ref.numbers((rows,), 6, F32, 0.1)
    w_lse, ln, w_h, mean_d = ref.softmax_parts(x)
    ws = workspace(zpp, rows, vocab)
    lp, lse, h = outputs(rows)
    zpp.log_probs_forward(x, targets, lp, lse, ws, entropies=h)
    check_forward(x, targets, lp, lse, h)
    top = min(vocab, 5)
    ids, tlp = torch.empty(rows, top, dtype=torch.int32, device="cuda"), torch.empty(rows, top, device="cuda")
    zpp.log_probs_forward(x, targets, lp, lse, workspace(zpp, rows, vocab, top), entropies=h,
                          top_ids=ids, top_log_probs=tlp)
    check_forward(x, targets, lp, lse, h)
    assert torch.equal(ids.long(), ref.top_ids(x, top))
    dx = torch.empty_like(x)
    zpp.log_probs_train(x, targets, lp, lse, g, dx, ws, entropies=h, dentropies=dh)
    check_forward(x, targets, lp, lse, h)
    if vocab <= 65536:  # (longer rows' second pass has lse as fp32 holds it)
        rel = ref.sum_bound(vocab, mean_d) + 2 * ref.U * (ln.abs() + 1)
        # relative to the row's largest logit, as the kernel takes them: no rounding of lse
        largest = x.double().amax(1)
        want, bound = ref.gradient(x.double() - largest[:, None], targets, ln, g, dh, w_h, rel_s=rel)
        assert_within(dx, want, bound)


# --------------------------------------------------------------------------
# Moments in 8 bits
# --------------------------------------------------------------------------
def tiny_moments(seed):
    """Blocks below the normal numbers, blocks whose largest is next to 2^-96 with denormals
    beside it, one value of many magnitudes, zeros of both signs, a negative one."""
    rng = np.random.default_rng(seed)
    x = np.abs(rng.standard_normal((12, 256))).astype(np.float32)
    x[0] *= np.float32(2.0 ** -140)
    x[1] *= np.float32(2.0 ** -98)
    x[2] *= np.float32(2.0 ** -97)
    x[3] *= np.float32(2.0 ** -126)
    x[3, 0] = 2.0 ** -96
    x[4] = 2.0 ** -149
    x[5] *= 2.0 ** np.float32(rng.integers(-60, 0, 256))
    x[6] = 0.0
    x[6, ::2] = -0.0
    x[7, 9] = -1.0
    x[8] = np.float32(2.0 ** -126)
    x[8, 1] = np.float32(2.0 ** -95)
    x[9] *= np.float32(2.0 ** 120)
    # squares of numbers on and beside the borders, at the scale of a largest root of 255^2
    c = np.arange(256) + 0.5
    for row, step in ((10, 0.0), (11, 2.0 ** -24)):
        x[row] = ((c[:256] ** 2 * (1 + step)) ** 2).astype(np.float32)
        x[row, 255] = 65025.0 ** 2
    return torch.from_numpy(x.reshape(-1)).cuda()


@pytest.mark.parametrize("moment", [1, 2])
def test_moments_next_to_every_edge(zpp, moment):
    x = tiny_moments(3)
    state = zpp.empty_adam_state(x.numel(), moment)
    zpp.adam_state_save(x, state)
    codes, scales = state8(x, moment)
    assert torch.equal(state[0], codes)
    assert same(state[1].nan_to_num(nan=-1), scales.nan_to_num(nan=-1))
    out = torch.empty_like(x)
    zpp.adam_state_load(state, out)
    assert same(out.nan_to_num(nan=-1), values8((codes, scales), moment).nan_to_num(nan=-1))


def test_many_seeds_of_moments(zpp):
    """Four million second moments: some thousand waves that take their codes from correct
    roots."""
    x = ref.numbers((1 << 22,), 9, F32).square_()
    state = zpp.empty_adam_state(x.numel(), 2)
    zpp.adam_state_save(x, state)
    codes, scales = state8(x, 2)
    assert torch.equal(state[0], codes) and same(state[1], scales)


# --------------------------------------------------------------------------
# A training step
# --------------------------------------------------------------------------
def test_a_step_of_a_model(zpp):
    """One layer of attention over a vocabulary: the fused product's queries and keys turned
    in place, the loss with its gradient in the logits' place, the way back, and the step
    of all weights.  Each operator's results against its 64-bit form on what it was given;
    the weights' bits as the step of one tensor makes them."""
    tokens, heads, kv, dim, vocab, hidden = 70, 4, 2, 32, 517, 96
    def weight(*shape, seed):
        return ref.numbers(shape, seed, F32, 0.1)

    w_qkv, w_out = weight(hidden, (heads + 2 * kv) * dim, seed=1), weight(heads * dim, vocab, seed=2)
    x = ref.numbers((tokens, hidden), 3, F32)
    gen = torch.Generator(device="cuda").manual_seed(4)
    targets = torch.randint(vocab, (tokens,), device="cuda", generator=gen)
    targets[::9] = -100
    positions, turns = plan(zpp, tokens, dim, 4000)

    qkv = (x @ w_qkv).view(tokens, heads + 2 * kv, dim)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    before = qkv.clone()
    zpp.rotary_forward(q, positions, turns, q, k=k, k_out=k)
    want, bound = ref.rotated(before[:, None, :heads + kv], positions, turns, False, 1.0, False)
    assert_within(qkv[:, None, :heads + kv], want, bound)
    assert same(v, before[:, heads + kv:])

    # attention and the head in torch, the heads' keys repeated
    leaf = qkv.detach().requires_grad_()
    rep = heads // kv
    qq = leaf[:, :heads].transpose(0, 1)
    kk = leaf[:, heads:heads + kv].repeat_interleave(rep, 1).permute(1, 2, 0).contiguous()
    vv = leaf[:, heads + kv:].repeat_interleave(rep, 1).transpose(0, 1).contiguous()
    mask = torch.full((tokens, tokens), -INF, device="cuda").triu(1)
    p = torch.softmax(qq.contiguous() @ kk / dim ** 0.5 + mask, -1)
    mixed = (p @ vv).transpose(0, 1).reshape(tokens, heads * dim)
    out = mixed @ w_out

    l = out.detach().clone()
    given = l.clone()
    g = torch.full((tokens,), -1.0 / tokens, device="cuda")
    (lp, lse, _), ws = outputs(tokens), workspace(zpp, tokens, vocab)
    zpp.log_probs_train(l, targets, lp, lse, g, l, ws)
    check_forward(given, targets, lp, lse, None)
    w_lse, ln, _, mean_d = ref.softmax_parts(given)
    want, bound = ref.gradient(given, targets, w_lse, g,
                               rel_s=ref.sum_bound(vocab, mean_d) + 2 * ref.U * (ln.abs() + 1))
    assert_within(l, want, bound)

    dqkv, = torch.autograd.grad(out, leaf, l)
    d_out = mixed.detach().t() @ l
    before = dqkv.clone()
    dq, dk = dqkv[:, :heads], dqkv[:, heads:heads + kv]
    zpp.rotary_backward(dq, positions, turns, dq, k=dk, k_out=dk)
    want, bound = ref.rotated(before[:, None, :heads + kv], positions, turns, False, 1.0, True)
    assert_within(dqkv[:, None, :heads + kv], want, bound)
    d_qkv = x.t() @ dqkv.reshape(tokens, -1)

    weights, grads = [w_qkv.view(-1), w_out.view(-1)], [d_qkv.view(-1), d_out.view(-1)]
    moments = [[torch.zeros_like(w) for w in weights] for _ in range(2)]
    copies = [torch.empty_like(w, dtype=BF16) for w in weights]
    one = [[t.clone() for t in x] for x in (weights, *moments)]
    tensors = zpp.AdamTensors(weights, *moments, grads, copies, weight_decay=[0.1, 0.0])
    zpp.adam_tensors_step(tensors, step=1, **HP)
    for i, decay in enumerate((0.1, 0.0)):
        copy = torch.empty_like(copies[i])
        zpp.adam_partition_step(one[0][i], one[1][i], one[2][i], grads[i].contiguous(), copy,
                                step=1, weight_decay=decay, **HP)
        assert same(weights[i], one[0][i]) and same(copies[i], copy)
        assert same(moments[0][i], one[1][i]) and same(moments[1][i], one[2][i])


def test_more_rows_than_a_launch_takes(zpp):
    """2^20 workgroups are a launch: the rows past them are a second one's."""
    rows, vocab = (1 << 20) + 77, 16
    x, targets = logits(rows, vocab, 0, BF16, 11)
    lp, lse, h = outputs(rows)
    ids = torch.empty(rows, 2, dtype=torch.int32, device="cuda")
    tlp = torch.empty(rows, 2, device="cuda")
    zpp.log_probs_forward(x, targets, lp, lse, workspace(zpp, rows, vocab, 2), entropies=h,
                          top_ids=ids, top_log_probs=tlp)
    check_forward(x, targets, lp, lse, h)
    assert torch.equal(ids.long(), ref.top_ids(x, 2))
