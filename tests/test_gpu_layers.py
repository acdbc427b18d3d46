"""The layer operators (layer norm, GELU, checkpoints in 8 bits, weight
gradient) on the GPU against plain 64-bit forms, with bounds derived in
tests/layer_reference.py: element types, odd sizes, strides and starts, rows of
one element and of more than fit registers, empty calls, NaN and Inf, gradients
against differences, streams, and the same bits on every run."""
import numpy as np
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def zpp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_01614_amd import zpp as mod
    return mod


# rows, cols, pad, offset: one element, less than a chunk, a block and one more,
# ragged ones, wide ones, more rows than workgroups
SIZES = [(1, 1, 0, 0), (3, 7, 1, 1), (5, 64, 0, 0), (2, 65, 3, 2), (17, 1001, 7, 1),
         (33, 512, 0, 8), (1, 4544, 0, 0), (130, 4544, 131, 3), (2100, 72, 0, 0),
         (7, 8192, 0, 0), (600, 520, 8, 0), (5, 8200, 1, 0), (3, 20000, 0, 1), (2, 40001, 3, 0)]
IDS = ["%dx%d+%d@%d" % s for s in SIZES]
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
EACH_SIZE = pytest.mark.parametrize("rows,cols,pad,offset", SIZES, ids=IDS)


def bits(t):
    return t.contiguous().view({2: torch.int16, 4: torch.int32, 1: torch.uint8}[t.element_size()])


def same(a, b):
    return torch.equal(bits(a), bits(b))


# --------------------------------------------------------------------------
# Checkpoints
# --------------------------------------------------------------------------
def hard_values(rows, cols, seed, dtype, pad=0, offset=0):
    """Values over the whole range: rows of every magnitude, largest elements on
    and beside 127 * 2^e, halves between codes, zeros, Inf and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-140, 127, (rows, 1))
    x[0::5] = rng.integers(-254, 255, x[0::5].shape) / 2.0      # halves: ties
    x[1::5, ::3] = 0
    x[2::7] = 127 * 2.0 ** rng.integers(-30, 30, x[2::7].shape)  # as large as a block takes
    x[3::11, cols // 2] = np.inf
    x[4::11, cols // 3] = np.nan
    x[5::11, 0] = 3.3895e38
    x = np.clip(x, -3.3895e38, 3.3895e38, where=np.isfinite(x), out=x)
    m = ref.matrix(rows, cols, dtype, pad, offset)
    m.copy_(torch.from_numpy(x.astype(np.float32)))
    return m


@TYPES
@EACH_SIZE
def test_checkpoint_save_and_load(zpp, rows, cols, pad, offset, dtype):
    x = hard_values(rows, cols, 11 * rows + cols, dtype, pad, offset)
    codes, exps = ref.encode(x.float().cpu().numpy())
    saved = (ref.matrix(rows, cols, torch.int8, pad, offset), torch.empty(
        rows, -(-cols // 64), dtype=torch.uint8, device="cuda"))
    zpp.checkpoint_save(x, saved)
    assert np.array_equal(saved[1].cpu().numpy(), exps)
    assert np.array_equal(saved[0].cpu().numpy(), codes)
    out = ref.matrix(rows, cols, dtype, pad + 2, offset)
    zpp.checkpoint_load(saved, out)
    want = torch.from_numpy(ref.decode(codes, exps)).cuda()
    got = out.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(), want.nan_to_num())
    # within half a step of a finite input
    finite = torch.isfinite(want) & torch.isfinite(x)
    step = torch.from_numpy(np.repeat(2.0 ** (exps.astype(np.float64) - 127), 64, 1)[:, :cols])
    low = want.abs() < 63 * 2.0 ** 122   # all but codes kept to 63
    far = (x.double() - want).abs() > step.cuda() / 2
    assert not (far & finite & low).any()


def test_checkpoint_keeps_what_is_beside_it(zpp):
    """Rows that lie apart: what is between them is not written."""
    x = ref.values(9, 77, 3, BF16)
    codes = ref.matrix(9, 77, torch.int8, 5, 3, fill=99)
    exps = torch.full((9 * 2 + 1,), 99, dtype=torch.uint8, device="cuda")
    zpp.checkpoint_save(x, (codes, exps[:18].view(9, 2)))
    around = codes.as_strided((9, 5), (82, 1), codes.storage_offset() + 77)
    assert bool((around[:8] == 99).all()) and int(exps[18]) == 99
    out = ref.matrix(9, 77, F32, 3, 1, fill=7.0)
    zpp.checkpoint_load((codes, exps[:18].view(9, 2)), out)
    assert bool((out.as_strided((8, 3), (80, 1), 1 + 77) == 7.0).all())


# --------------------------------------------------------------------------
# Layer norm
# --------------------------------------------------------------------------
def norm_params(cols, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    g = (1 + 0.3 * torch.randn(cols, device="cuda", generator=gen)).to(dtype)
    b = (0.3 * torch.randn(cols, device="cuda", generator=gen)).to(dtype)
    return g, b


@pytest.mark.parametrize("params", [BF16, F32], ids=["pbf16", "pf32"])
@TYPES
@EACH_SIZE
def test_norm_forward(zpp, rows, cols, pad, offset, dtype, params):
    eps = 1e-5
    x = ref.values(rows, cols, 1, dtype, pad, offset)
    x.add_(3.0)
    gamma, beta = norm_params(cols, params, 2)
    want, bound = ref.norm_forward(x.double(), gamma.double(), beta.double(), eps, dtype)
    y = ref.matrix(rows, cols, dtype, pad, 2)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=eps)
    for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
        ref.check(got, w, b, what)
    # without a bias, and with nothing kept for a backward pass
    again = ref.matrix(rows, cols, dtype)
    zpp.layer_norm_forward(x, gamma, None, again, None, None, eps=eps)
    want, bound = ref.norm_forward(x.double(), gamma.double(), torch.zeros_like(beta).double(),
                                   eps, dtype)
    ref.check(again, want[0], bound[0], "y without a bias")


@TYPES
@EACH_SIZE
def test_norm_forward_with_residual_and_checkpoint(zpp, rows, cols, pad, offset, dtype):
    eps = 1e-6
    x = ref.values(rows, cols, 4, dtype, pad, offset)
    r = ref.values(rows, cols, 5, dtype, pad + 1, 0, std=2.0)
    gamma, beta = norm_params(cols, F32, 6)
    y, total = ref.matrix(rows, cols, dtype), ref.matrix(rows, cols, dtype, pad, 1)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    saved = zpp.empty_checkpoint(rows, cols)
    zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=eps, residual=r, total=total,
                           saved=saved)
    assert same(total, (x.float() + r.float()).to(dtype))
    want, bound = ref.norm_forward(total.double(), gamma.double(), beta.double(), eps, dtype)
    for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
        ref.check(got, w, b, what)
    codes, exps = ref.encode(total.float().cpu().numpy())
    assert np.array_equal(saved[0].cpu().numpy(), codes)
    assert np.array_equal(saved[1].cpu().numpy(), exps)


@pytest.mark.parametrize("again", [False, True], ids=["", "y"])
@pytest.mark.parametrize("from_saved", [False, True], ids=["plain", "i8"])
@TYPES
@EACH_SIZE
def test_norm_backward(zpp, rows, cols, pad, offset, dtype, from_saved, again):
    x = ref.values(rows, cols, 7, dtype, pad, offset)
    dy = ref.values(rows, cols, 8, dtype, pad, 1, std=1e-3)
    dres = ref.values(rows, cols, 9, dtype, 0, offset, std=1e-3) if again else None
    gamma, beta = norm_params(cols, F32 if from_saved else dtype, 10)
    mean = x.float().mean(1)
    rstd = torch.rsqrt((x.float() - mean[:, None]).square().mean(1) + 1e-5)
    arg, xs = ref.saved(x) if from_saved else (x, x.double())
    want, bound = ref.norm_backward(dy.double(), xs, gamma.double(), beta.double(), mean.double(),
                                    rstd.double(), None if dres is None else dres.double(), dtype)
    dx = ref.matrix(rows, cols, dtype, pad, offset)
    y = ref.matrix(rows, cols, dtype, 3, 0) if again else None
    dg, db = torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    ws = torch.empty(zpp.layer_norm_backward_workspace(rows, cols), dtype=torch.uint8,
                     device="cuda").fill_(0xFF)
    zpp.layer_norm_backward(dy, arg, gamma, mean, rstd, dx, dg, db, ws, dresidual=dres,
                            beta=beta if again else None, y=y)
    for got, w, b, what in zip((dx, dg, db, y), want, bound, ("dx", "dgamma", "dbeta", "y")):
        if got is not None:
            ref.check(got, w, b, what)
    # added to what is there: one more rounding of the sum
    ag, ab = dg.clone(), db.clone()
    once = dx.clone()
    zpp.layer_norm_backward(dy, arg, gamma, mean, rstd, dx, ag, ab, ws, dresidual=dres,
                            beta=beta if again else None, y=y, accumulate=True)
    assert same(dx, once) and same(ag, dg + dg) and same(ab, db + db)
    # frozen weights
    dx.fill_(0)
    zpp.layer_norm_backward(dy, arg, gamma, mean, rstd, dx, None, None, ws, dresidual=dres)
    assert same(dx, once)


def test_norm_of_constant_rows(zpp):
    """No variance: rstd is 1 / sqrt(eps), y the bias, also of large values."""
    for value in (0.0, 1.0, -300.0):
        x = torch.full((4, 1000), value, device="cuda")
        gamma, beta = norm_params(1000, F32, 1)
        y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), \
            torch.empty(4, device="cuda")
        zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=1e-5)
        want, bound = ref.norm_forward(x.double(), gamma.double(), beta.double(), 1e-5, F32)
        for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
            ref.check(got, w, b, what)


def test_norm_nan_stays_in_its_row(zpp):
    x = ref.values(6, 300, 2, BF16)
    x[1, 17] = float("nan")
    x[4, 250] = float("inf")
    gamma, beta = norm_params(300, BF16, 1)
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    saved = zpp.empty_checkpoint(6, 300)
    zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=1e-5, saved=saved)
    rows = torch.tensor([False, True, False, False, True, False])
    assert torch.equal(torch.isnan(y).all(1).cpu(), rows)
    assert torch.equal(torch.isnan(y).any(1).cpu(), rows)
    assert int((saved[1] == 255).sum()) == 2
    ok = ref.values(6, 300, 2, BF16)
    dx, dg, db = torch.empty_like(x), torch.empty(300, device="cuda"), \
        torch.empty(300, device="cuda")
    ws = torch.empty(zpp.layer_norm_backward_workspace(6, 300), dtype=torch.uint8, device="cuda")
    zpp.layer_norm_backward(ok, saved, gamma, mean, rstd, dx, dg, db, ws)
    assert torch.equal(torch.isnan(dx).any(1).cpu(), rows)
    assert bool(torch.isfinite(db).all()) and bool(torch.isnan(dg).any())


def test_norm_backward_against_differences(zpp):
    """The gradient of sum(w y) by x, gamma and beta, against central differences
    of the 64-bit forward pass (their own error: h^2 of the third derivative)."""
    rows, cols, eps, h = 3, 37, 1e-5, 1e-4
    x, w = ref.values(rows, cols, 1, F32), ref.values(rows, cols, 2, F32)
    gamma, beta = norm_params(cols, F32, 3)

    def loss(x, g, b):
        (y, _, _), _ = ref.norm_forward(x, g, b, eps, F32)
        return float((y * w.double()).sum())

    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), \
        torch.empty(rows, device="cuda")
    zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=eps)
    dx, dg, db = torch.empty_like(x), torch.empty(cols, device="cuda"), \
        torch.empty(cols, device="cuda")
    ws = torch.empty(zpp.layer_norm_backward_workspace(rows, cols), dtype=torch.uint8,
                     device="cuda")
    zpp.layer_norm_backward(w, x, gamma, mean, rstd, dx, dg, db, ws)
    args = [x.double(), gamma.double(), beta.double()]
    for i, got in enumerate((dx, dg, db)):
        for at in range(0, args[i].numel(), 5):
            d = torch.zeros_like(args[i]).view(-1)
            d[at] = h
            d = d.view_as(args[i])
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + d, args[i] - d
            diff = (loss(*up) - loss(*down)) / (2 * h)
            assert abs(float(got.view(-1)[at]) - diff) < 2e-5 * max(1.0, abs(diff)), (i, at)


# --------------------------------------------------------------------------
# GELU
# --------------------------------------------------------------------------
@pytest.mark.parametrize("from_saved", [False, True], ids=["plain", "i8"])
@TYPES
@EACH_SIZE
def test_gelu(zpp, rows, cols, pad, offset, dtype, from_saved):
    u = ref.values(rows, cols, 1, dtype, pad, offset, std=3.0)
    da = ref.values(rows, cols, 2, dtype, pad, 1, std=1e-3)
    (a, _), (ba, _) = ref.gelu(u.double(), da.double(), dtype)
    out = ref.matrix(rows, cols, dtype, pad, offset)
    saved = zpp.empty_checkpoint(rows, cols) if from_saved else None
    zpp.gelu_forward(u, out, saved=saved)
    ref.check(out, a, ba, "a")
    x = u.double()
    if from_saved:
        codes, exps = ref.encode(u.float().cpu().numpy())
        assert np.array_equal(saved[0].cpu().numpy(), codes)
        assert np.array_equal(saved[1].cpu().numpy(), exps)
        x = torch.from_numpy(ref.decode(codes, exps)).cuda()
    (a, du), (ba, bd) = ref.gelu(x, da.double(), dtype)
    got, again = ref.matrix(rows, cols, dtype, 1, 0), ref.matrix(rows, cols, dtype, pad, 3)
    zpp.gelu_backward(da, saved if from_saved else u, got, a=again)
    ref.check(got, du, bd, "du")
    ref.check(again, a, ba, "a again")
    alone = ref.matrix(rows, cols, dtype)
    zpp.gelu_backward(da, saved if from_saved else u, alone)
    assert same(alone, got)


def test_gelu_over_its_whole_range(zpp):
    """Every bf16 number, and the 32-bit form between: infinities and the tail
    take their limits, NaN stays."""
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(BF16)
    for u, dtype in ((every.view(256, 256), BF16),
                     (torch.linspace(-20, 20, 60000, device="cuda").view(60, 1000), F32)):
        one = torch.ones_like(u)
        a, du = torch.empty_like(u), torch.empty_like(u)
        zpp.gelu_forward(u, a)
        zpp.gelu_backward(one, u, du)
        x = u.double()
        nan = torch.isnan(x)
        assert torch.equal(torch.isnan(a), nan) and torch.equal(torch.isnan(du), nan)
        inside = x.abs() < 1e3
        (wa, wd), (ba, bd) = ref.gelu(torch.where(inside, x, torch.zeros_like(x)), one.double(),
                                      dtype)
        keep = inside & ~nan
        ref.check(a[keep], wa[keep], ba[keep], "a")
        ref.check(du[keep], wd[keep], bd[keep], "du")
        far = ~inside & ~nan
        assert torch.equal(a[far].double(), torch.where(x > 0, x, torch.zeros_like(x))[far])
        assert torch.equal(du[far].double(), (x > 0).double()[far])


def test_gelu_backward_against_differences(zpp):
    u = torch.linspace(-6, 6, 1001, device="cuda").view(7, 143)
    du = torch.empty_like(u)
    zpp.gelu_backward(torch.ones_like(u), u, du)
    h = 1e-4
    f = lambda x: x * 0.5 * torch.special.erfc(-x * 0.5 ** 0.5)
    diff = (f(u.double() + h) - f(u.double() - h)) / (2 * h)
    # h^2 / 6 of the third derivative, which stays below 2, and the kernel's bound
    assert float((du.double() - diff).abs().max()) < h * h + 4e-7


# --------------------------------------------------------------------------
# Weight gradient
# --------------------------------------------------------------------------
GRADS = [(1, 1, 1), (1, 64, 64), (3, 5, 130), (63, 128, 128), (64, 129, 127), (65, 256, 64),
         (77, 1000, 777), (200, 257, 520), (500, 40, 300), (2000, 128, 192), (4099, 72, 200),
         (130, 513, 1025), (300, 1030, 260)]


def run_grad(zpp, dy, x, n, k, **kw):
    rows = dy.shape[0]
    dw = ref.matrix(n, k, F32, fill=7.0)
    ws = torch.empty(zpp.weight_grad_workspace(rows, n, k), dtype=torch.uint8,
                     device="cuda").fill_(0xFF)
    zpp.weight_grad(dy, x, dw, ws, **kw)
    return dw


@pytest.mark.parametrize("from_saved", [False, True], ids=["bf16", "i8"])
@pytest.mark.parametrize("rows,n,k", GRADS, ids=["%dx%dx%d" % g for g in GRADS])
@pytest.mark.parametrize("pad,offset", [(0, 0), (5, 3), (8, 8)], ids=["dense", "odd", "wide"])
def test_weight_grad(zpp, rows, n, k, pad, offset, from_saved):
    dy = ref.values(rows, n, 1, BF16, pad, offset, std=1e-3)
    x = ref.values(rows, k, 2, BF16, pad, offset)
    arg, xs = ref.saved(x) if from_saved else (x, x.double())
    want, bound = ref.weight_grad(dy.double(), xs)
    dw = run_grad(zpp, dy, arg, n, k)
    ref.check(dw, want, bound, "dw")
    # added to a gradient whose rows lie apart: what is between stays
    wide = ref.matrix(n, k, F32, 3, 1, fill=0.5)
    ws = torch.empty(zpp.weight_grad_workspace(rows, n, k), dtype=torch.uint8, device="cuda")
    zpp.weight_grad(dy, arg, wide, ws, accumulate=True)
    ref.check(wide, want + 0.5, bound + 2 * ref.U * (want.abs() + 0.5), "dw added to")
    if n > 1:
        between = wide.as_strided((n - 1, 3), (k + 3, 1), 1 + k)
        assert bool((between == 0.5).all())


def test_weight_grad_takes_exact_products(zpp):
    """Values whose products and sums 32 bits hold exactly: no rounding at all,
    also from a checkpoint (its elements reach the products unrounded)."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    dy = torch.randint(-8, 9, (300, 200), device="cuda", generator=gen).to(BF16)
    x = torch.randint(-127, 128, (300, 330), device="cuda", generator=gen).to(BF16)
    want = dy.double().t() @ x.double()
    saved = zpp.empty_checkpoint(300, 330)
    zpp.checkpoint_save(x, saved)
    assert torch.equal(run_grad(zpp, dy, x, 200, 330).double(), want)
    assert torch.equal(run_grad(zpp, dy, saved, 200, 330).double(), want)


def test_weight_grad_nan_and_inf(zpp):
    """A NaN reaches its row or column of dw alone: padding of a tile's ends is
    zeros, not what lies past the rows."""
    rows, n, k = 70, 140, 90
    big = ref.values(128, 256, 1, BF16)
    dy, x = big[:rows, :n], ref.values(128, 256, 2, BF16)
    x[rows:] = float("nan")
    x[:, k:] = float("nan")
    big[rows:] = float("nan")
    big[:, n:] = float("inf")
    x = x[:rows, :k]
    assert bool(torch.isfinite(run_grad(zpp, dy, x, n, k)).all())
    dy[69, 7] = float("nan")
    x[3, 80] = float("inf")
    dw = torch.isfinite(run_grad(zpp, dy, x, n, k))
    want = torch.ones(n, k, dtype=torch.bool, device="cuda")
    want[7] = False
    want[:, 80] = False
    assert torch.equal(dw, want)
    saved = zpp.empty_checkpoint(rows, k)
    zpp.checkpoint_save(x, saved)
    want[:, 64:] = False   # the block that holds the Inf reads as NaN
    assert torch.equal(torch.isfinite(run_grad(zpp, dy, saved, n, k)), want)


def test_weight_grad_against_differences(zpp):
    """The gradient of sum(dy * x W^T), linear in W: differences are exact."""
    rows, n, k = 9, 5, 11
    dy, x = ref.values(rows, n, 1, BF16), ref.values(rows, k, 2, BF16)
    dw = run_grad(zpp, dy, x, n, k)
    w = torch.zeros(n, k, dtype=torch.float64, device="cuda")
    loss = lambda w: float((dy.double() * (x.double() @ w.t())).sum())
    for i in range(n):
        for j in range(k):
            w[i, j] = 1.0
            assert abs(float(dw[i, j]) - loss(w)) < 1e-5
            w[i, j] = 0.0


# --------------------------------------------------------------------------
# All of them
# --------------------------------------------------------------------------
def test_empty_calls(zpp):
    """No rows or no features: nothing is read or written but the gradients of
    weights, which are sums of nothing; events are recorded."""
    f = lambda *s: torch.empty(*s, device="cuda")
    ev = zpp.Event()
    none = zpp.empty_checkpoint(0, 64)
    zpp.checkpoint_save(f(0, 64), none, done_after=ev)
    ev.synchronize()
    zpp.checkpoint_load(none, f(0, 64))
    zpp.checkpoint_save(f(3, 0), zpp.empty_checkpoint(3, 0))
    zpp.gelu_forward(f(0, 64), f(0, 64))
    zpp.gelu_backward(f(0, 64), none, f(0, 64))
    g = torch.ones(64, device="cuda")
    zpp.layer_norm_forward(f(0, 64), g, g, f(0, 64), f(0), f(0), eps=1e-5)
    dg, db = torch.full((64,), 3.0, device="cuda"), torch.full((64,), 4.0, device="cuda")
    for add, left in ((True, (3.0, 4.0)), (False, (0.0, 0.0))):
        zpp.layer_norm_backward(f(0, 64), none, g, f(0), f(0), f(0, 64), dg, db, None,
                                accumulate=add)
        assert bool((dg == left[0]).all()) and bool((db == left[1]).all())
    dw = torch.full((64, 70), 3.0, device="cuda")
    b = lambda *s: torch.empty(*s, dtype=BF16, device="cuda")
    for add, left in ((True, 3.0), (False, 0.0)):
        zpp.weight_grad(b(0, 64), b(0, 70), dw, None, accumulate=add)
        assert bool((dw == left).all())
    zpp.weight_grad(b(5, 0), b(5, 70), f(0, 70), None)


def layer_pass(zpp, x, dy, w, gamma, beta, dw, bufs, stream=None, wait=None, done=None):
    """A norm, GELU and weight gradient through checkpoints, as one sequence."""
    b = bufs
    zpp.layer_norm_forward(x, gamma, beta, b["y"], b["mean"], b["rstd"], eps=1e-5,
                           saved=b["x8"], stream=stream, wait_before=wait)
    zpp.gelu_forward(b["y"], b["a"], saved=b["y8"], stream=stream)
    zpp.gelu_backward(dy, b["y8"], b["du"], a=b["a2"], stream=stream)
    zpp.layer_norm_backward(b["du"], b["x8"], gamma, b["mean"], b["rstd"], b["dx"], b["dg"],
                            b["db"], b["ws"], beta=beta, y=b["y2"], stream=stream)
    zpp.weight_grad(dy, b["y8"], dw, b["wws"], stream=stream, done_after=done)


def layer_buffers(zpp, rows, cols):
    m = lambda: ref.matrix(rows, cols, BF16)
    v = lambda n: torch.empty(n, device="cuda")
    ws = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    return dict(y=m(), a=m(), a2=m(), y2=m(), du=m(), dx=m(), mean=v(rows), rstd=v(rows),
                dg=v(cols), db=v(cols), x8=zpp.empty_checkpoint(rows, cols),
                y8=zpp.empty_checkpoint(rows, cols),
                ws=ws(zpp.layer_norm_backward_workspace(rows, cols)),
                wws=ws(zpp.weight_grad_workspace(rows, cols, cols)))


def flat(bufs, dw):
    out = [dw]
    for k, v in sorted(bufs.items()):
        if k not in ("ws", "wws"):
            out += list(v) if isinstance(v, tuple) else [v]
    return [bits(t).clone() for t in out]


def test_same_bits_on_every_run_stream_and_replay(zpp):
    """The sequence twice, on a stream of its own behind an event, and replayed
    from a graph with eager work between: the same bits each time."""
    rows, cols = 700, 1000
    x, dy = ref.values(rows, cols, 1, BF16), ref.values(rows, cols, 2, BF16, std=1e-3)
    gamma, beta = norm_params(cols, BF16, 3)
    dw = torch.empty(cols, cols, device="cuda")
    bufs = layer_buffers(zpp, rows, cols)
    layer_pass(zpp, x, dy, None, gamma, beta, dw, bufs)
    torch.cuda.synchronize()
    first = flat(bufs, dw)

    def poison():
        for t in [dw] + [t for v in bufs.values() for t in (v if isinstance(v, tuple) else (v,))]:
            bits(t).fill_(0x55) if t.is_contiguous() else t.fill_(7)

    def expect(what):
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(first, flat(bufs, dw))):
            assert torch.equal(a, b), (what, i)

    poison()
    layer_pass(zpp, x, dy, None, gamma, beta, dw, bufs)
    expect("again")
    poison()
    side, ready, done = torch.cuda.Stream(), zpp.Event(), zpp.Event()
    ready.record()
    layer_pass(zpp, x, dy, None, gamma, beta, dw, bufs, stream=side, wait=ready, done=done)
    done.synchronize()
    expect("another stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer_pass(zpp, x, dy, None, gamma, beta, dw, bufs)
    for i in range(3):
        poison()
        torch.cuda.synchronize()
        graph.replay()
        expect("replay %d" % i)


def test_offsets_past_32_bits(zpp):
    """Rows that lie 2^31 and more bytes apart."""
    rows, cols, apart = 3, 200, (1 << 30) + 24
    buf = torch.empty(2 * apart + cols, dtype=BF16, device="cuda")
    far = buf.as_strided((rows, cols), (apart, 1))
    near = ref.values(rows, cols, 1, BF16)
    far.copy_(near)
    dy = ref.values(rows, cols, 2, BF16, std=1e-3)
    gamma, beta = norm_params(cols, F32, 3)
    got = {}
    for name, x in (("near", near), ("far", far)):
        b = layer_buffers(zpp, rows, cols)
        dw = torch.empty(cols, cols, device="cuda")
        layer_pass(zpp, x, dy, None, gamma, beta, dw, b)
        zpp.weight_grad(x, x, dw, b["wws"])
        zpp.gelu_backward(x, x, b["du"])
        got[name] = flat(b, dw)
    for a, b in zip(got["near"], got["far"]):
        assert torch.equal(a, b)
    # and as outputs
    far.fill_(7)
    saved = zpp.empty_checkpoint(rows, cols)
    zpp.checkpoint_save(near, saved)
    zpp.checkpoint_load(saved, far)
    out = torch.empty_like(near)
    zpp.checkpoint_load(saved, out)
    assert same(far, out)
    zpp.gelu_forward(near, far)
    zpp.gelu_forward(near, out)
    assert same(far, out)


# Rows of two chunks a lane in the norm's forward pass, ragged and not, the last
# length in registers and the first beyond
@TYPES
@pytest.mark.parametrize("rows,cols", [(3, 9001), (600, 16384), (2, 16383), (2, 16385), (4, 5)])
def test_norm_of_long_and_of_tiny_rows(zpp, rows, cols, dtype):
    eps = 1e-5
    x, r = ref.values(rows, cols, 1, dtype, 3, 1), ref.values(rows, cols, 2, dtype)
    gamma, beta = norm_params(cols, dtype, 3)
    y, total = ref.matrix(rows, cols, dtype, 1), ref.matrix(rows, cols, dtype)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    saved = zpp.empty_checkpoint(rows, cols)
    zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=eps, residual=r, total=total,
                           saved=saved)
    want, bound = ref.norm_forward(total.double(), gamma.double(), beta.double(), eps, dtype)
    for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
        ref.check(got, w, b, what)
    codes, exps = ref.encode(total.float().cpu().numpy())
    assert np.array_equal(saved[0].cpu().numpy(), codes)
    assert np.array_equal(saved[1].cpu().numpy(), exps)
    dy = ref.values(rows, cols, 4, dtype, std=1e-3)
    xs = torch.from_numpy(ref.decode(codes, exps)).cuda()
    want, bound = ref.norm_backward(dy.double(), xs, gamma.double(), beta.double(), mean.double(),
                                    rstd.double(), None, dtype)
    dx, dg, db = ref.matrix(rows, cols, dtype), torch.empty(cols, device="cuda"), \
        torch.empty(cols, device="cuda")
    ws = torch.empty(zpp.layer_norm_backward_workspace(rows, cols), dtype=torch.uint8,
                     device="cuda")
    zpp.layer_norm_backward(dy, saved, gamma, mean, rstd, dx, dg, db, ws)
    for got, w, b, what in zip((dx, dg, db), want, bound, ("dx", "dgamma", "dbeta")):
        ref.check(got, w, b, what)


# Sizes for each way the weight gradient divides its work: tiles of 256 whole,
# a last round split over the tokens, few tiles split, at a multiple of the
# turn of 64 tokens and off it
@pytest.mark.parametrize("from_saved", [False, True], ids=["bf16", "i8"])
@pytest.mark.parametrize("rows,n,k", [(256, 4100, 4096), (641, 4672, 4544), (320, 4096, 4608),
                                      (2047, 300, 520), (4096, 256, 256)])
def test_weight_grad_divisions(zpp, rows, n, k, from_saved):
    dy, x = ref.values(rows, n, 1, BF16, std=1e-3), ref.values(rows, k, 2, BF16)
    saved = zpp.empty_checkpoint(rows, k)
    zpp.checkpoint_save(x, saved)
    xs = x.float()
    if from_saved:
        xs = torch.empty_like(xs)
        zpp.checkpoint_load(saved, xs)
    want, bound = ref.weight_grad(dy.double(), xs.double())
    dw = run_grad(zpp, dy, saved if from_saved else x, n, k)
    ref.check(dw, want, bound, "dw")
    assert same(dw, run_grad(zpp, dy, saved if from_saved else x, n, k))
    ws = torch.empty(zpp.weight_grad_workspace(rows, n, k), dtype=torch.uint8, device="cuda")
    twice = dw.clone()
    zpp.weight_grad(dy, saved if from_saved else x, twice, ws, accumulate=True)
    ref.check(twice, 2 * want, 2 * bound + 2 * ref.U * want.abs(), "dw added to")


def test_weight_grad_of_tokens_far_apart(zpp):
    """Tokens further apart than a turn's 32-bit offsets reach, more than one turn
    of them."""
    rows, n, k, apart = 70, 40, 72, (1 << 24) + 8
    buf = torch.empty(69 * apart + n, dtype=BF16, device="cuda")
    dy = buf.as_strided((rows, n), (apart, 1))
    near, x = ref.values(rows, n, 1, BF16), ref.values(rows, k, 2, BF16)
    dy.copy_(near)
    assert same(run_grad(zpp, dy, x, n, k), run_grad(zpp, near, x, n, k))


# Two chunks a lane, several rows a workgroup: the next row fetched while one is
# summed, partial last chunks among them
@TYPES
@pytest.mark.parametrize("rows,cols,pad", [(700, 8201, 0), (531, 14847, 3), (513, 12288, 1)])
def test_norm_forward_of_many_long_rows(zpp, rows, cols, pad, dtype):
    eps = 1e-5
    x, r = ref.values(rows, cols, 1, dtype, pad), ref.values(rows, cols, 2, dtype)
    gamma, beta = norm_params(cols, dtype, 3)
    y, total = ref.matrix(rows, cols, dtype, pad), ref.matrix(rows, cols, dtype)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    saved = zpp.empty_checkpoint(rows, cols)
    zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=eps, residual=r, total=total,
                           saved=saved)
    assert torch.equal(total, (x.float() + r.float()).to(dtype))
    want, bound = ref.norm_forward(total.double(), gamma.double(), beta.double(), eps, dtype)
    for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
        ref.check(got, w, b, what)
    codes, exps = ref.encode(total.float().cpu().numpy())
    assert np.array_equal(saved[0].cpu().numpy(), codes)
    assert np.array_equal(saved[1].cpu().numpy(), exps)


@pytest.mark.parametrize("again", [False, True], ids=["plain", "again"])
@pytest.mark.parametrize("from_saved", [False, True], ids=["same", "i8"])
@TYPES
@pytest.mark.parametrize("rows,cols,pad", [(1, 8208, 0), (700, 8201, 3), (300, 14847, 0),
                                           (513, 12288, 1)])
def test_norm_backward_of_long_rows(zpp, rows, cols, pad, dtype, from_saved, again):
    """Two chunks a lane, from one row to several a workgroup."""
    x = ref.values(rows, cols, 7, dtype, pad)
    dy = ref.values(rows, cols, 8, dtype, pad, std=1e-3)
    dres = ref.values(rows, cols, 9, dtype, std=1e-3) if again else None
    gamma, beta = norm_params(cols, F32 if from_saved else dtype, 10)
    mean = x.float().mean(1)
    rstd = torch.rsqrt((x.float() - mean[:, None]).square().mean(1) + 1e-5)
    arg, xs = ref.saved(x) if from_saved else (x, x.double())
    want, bound = ref.norm_backward(dy.double(), xs, gamma.double(), beta.double(), mean.double(),
                                    rstd.double(), None if dres is None else dres.double(), dtype)
    dx = ref.matrix(rows, cols, dtype, pad, fill=5.0)
    y = ref.matrix(rows, cols, dtype, 3) if again else None
    dg, db = torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    ws = torch.empty(zpp.layer_norm_backward_workspace(rows, cols), dtype=torch.uint8,
                     device="cuda").fill_(0xFF)
    zpp.layer_norm_backward(dy, arg, gamma, mean, rstd, dx, dg, db, ws, dresidual=dres,
                            beta=beta if again else None, y=y)
    for got, w, b, what in zip((dx, dg, db, y), want, bound, ("dx", "dgamma", "dbeta", "y")):
        if got is not None:
            ref.check(got, w, b, what)
    if pad and rows > 1:
        gaps = dx.as_strided((rows - 1, pad), (cols + pad, 1), dx.storage_offset() + cols)
        assert bool((gaps == 5.0).all())
    ag, ab, once = dg.clone(), db.clone(), dx.clone()
    zpp.layer_norm_backward(dy, arg, gamma, mean, rstd, dx, ag, ab, ws, dresidual=dres,
                            beta=beta if again else None, y=y, accumulate=True)
    assert same(dx, once) and same(ag, dg + dg) and same(ab, db + db)


@TYPES
def test_norm_backward_of_long_rows_keeps_a_rows_infinity_to_itself(zpp, dtype):
    """A row whose last element has no value: no other row's dx changes, and of the
    weights' gradients that column alone."""
    rows, cols = 5, 8201
    x, dy = ref.values(rows, cols, 7, dtype), ref.values(rows, cols, 8, dtype, std=1e-3)
    gamma, _ = norm_params(cols, dtype, 10)
    mean = x.float().mean(1)
    rstd = torch.rsqrt((x.float() - mean[:, None]).square().mean(1) + 1e-5)
    ws = torch.empty(zpp.layer_norm_backward_workspace(rows, cols), dtype=torch.uint8,
                     device="cuda")
    results = []
    for value in (0.5, float("inf"), float("nan")):
        x[2, cols - 1] = value
        dx, dg, db = ref.matrix(rows, cols, dtype), torch.empty(cols, device="cuda"), \
            torch.empty(cols, device="cuda")
        zpp.layer_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db, ws)
        results.append((dx, dg, db))
    clean = results[0]
    others = [0, 1, 3, 4]
    for dx, dg, db in results[1:]:
        assert same(dx[others].contiguous(), clean[0][others].contiguous())
        assert same(dg[:-1], clean[1][:-1]) and same(db, clean[2])
        assert not bool(torch.isfinite(dg[-1]))
        assert not bool(torch.isfinite(dx[2]).any())


# Rows of dw that end inside a tile's group of eight, at its edge, and inside the
# lower half of a tile; added to what is there, in rows that lie apart
@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("n,k", [(3, 5), (12, 130), (136, 8), (205, 33), (1000, 777), (259, 300)])
def test_weight_grad_adds_at_ragged_ends(zpp, rows, n, k):
    dy, x = ref.values(rows, n, 1, BF16, std=1e-3), ref.values(rows, k, 2, BF16)
    want, bound = ref.weight_grad(dy.double(), x.double())
    dw = ref.matrix(n, k, F32, 3, 1, fill=9.0)
    ws = torch.empty(zpp.weight_grad_workspace(rows, n, k), dtype=torch.uint8, device="cuda")
    zpp.weight_grad(dy, x, dw, ws)
    ref.check(dw, want, bound, "dw")
    once = dw.clone()
    before = torch.randn(n, k, device="cuda")
    dw.copy_(before)
    zpp.weight_grad(dy, x, dw, ws, accumulate=True)
    # one rounding of the same sum and what was there
    assert same(dw, before + once)
    if n > 1:
        gaps = dw.as_strided((n - 1, 3), (k + 3, 1), dw.storage_offset() + k)
        assert bool((gaps == 9.0).all())


@TYPES
@pytest.mark.parametrize("cols", [1, 3, 4, 5, 7, 8, 9, 28, 31, 32, 33, 35, 36, 37, 60, 63, 65, 92,
                                  95, 96, 97, 100, 127])
def test_each_end_of_a_block(zpp, cols, dtype):
    """Rows that end at every kind of place in a lane's share of a block: results to
    the last element, and nothing beyond it written."""
    rows, pad = 7, 5
    x = hard_values(rows, cols, cols, dtype, pad, 1)
    codes, exps = ref.encode(x.float().cpu().numpy())
    saved = (ref.matrix(rows, cols, torch.int8, pad, 3, fill=99),
             torch.empty(rows, -(-cols // 64), dtype=torch.uint8, device="cuda"))
    out, again = (ref.matrix(rows, cols, dtype, pad, 1, fill=7.0) for _ in range(2))
    u = ref.values(rows, cols, 5, dtype, pad)
    da = ref.values(rows, cols, 6, dtype, std=1e-3)
    a, du = (ref.matrix(rows, cols, dtype, pad, 2, fill=7.0) for _ in range(2))
    arg, us = ref.saved(u)
    zpp.checkpoint_save(x, saved)
    zpp.checkpoint_load(saved, out)
    zpp.gelu_forward(u, a)
    zpp.gelu_backward(da, arg, du, a=again)
    assert np.array_equal(saved[0].cpu().numpy(), codes)
    assert np.array_equal(saved[1].cpu().numpy(), exps)
    want = torch.from_numpy(ref.decode(codes, exps)).cuda().to(dtype)
    assert torch.equal(out.nan_to_num(), want.nan_to_num())
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    (wa, _), (ba, _) = ref.gelu(u.double(), da.double(), dtype)
    ref.check(a, wa, ba, "a")
    (wa, wd), (ba, bd) = ref.gelu(us, da.double(), dtype)
    ref.check(again, wa, ba, "a again")
    ref.check(du, wd, bd, "du")
    for m, was in ((saved[0], 99), (out, 7.0), (a, 7.0), (du, 7.0), (again, 7.0)):
        gaps = m.as_strided((rows - 1, pad), (cols + pad, 1), m.storage_offset() + cols)
        assert bool((gaps == was).all())
