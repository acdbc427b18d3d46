"""Layer norm's mean and variance of rows that hardly vary: the mean of a row is
known to its last bit, or a row of one value would not give its bias.  Against
plain 64-bit forms, with bounds from the roundings of a mean that is corrected by
the mean of the differences from it (U and `chain` of tests/layer_reference.py)."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U = ref.U
# long rows, rows of less than a chunk, whole and partial chunks, one and two a lane
COLS = [5, 64, 100, 1000, 1001, 3584, 4544, 8200, 8201, 12000, 20000]


@pytest.fixture(scope="module")
def zpp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_01614_amd import zpp as mod
    return mod


def params(cols):
    gen = torch.Generator(device="cuda").manual_seed(cols)
    return (1 + 0.3 * torch.randn(cols, device="cuda", generator=gen),
            0.3 * torch.randn(cols, device="cuda", generator=gen))


def forward(zpp, x, gamma, beta, eps):
    y = torch.empty_like(x)
    mean, rstd = torch.empty(len(x), device="cuda"), torch.empty(len(x), device="cuda")
    zpp.layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=eps)
    return y, mean, rstd


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("cols", COLS)
def test_rows_of_one_value(zpp, cols, dtype, eps):
    """The mean is the value and y the bias, both exactly: the first mean is off by
    (chain + 2) U of the value at most, its correction by as much of itself, so
    their sum is the value to less than half of its last bit.  What rounding leaves
    of the variance, the difference of two squares of the correction, is below
    3 (chain + 4) U of that square."""
    gamma, beta = params(cols)
    values = torch.tensor([0.0, 1.0, 700.0, 0.1, -3.7e5, 10000 / 3, -5e-20], device="cuda")
    values = values.to(dtype).float()
    x = values.to(dtype)[:, None].expand(-1, cols).contiguous()
    y, mean, rstd = forward(zpp, x, gamma, beta, eps)
    assert torch.equal(mean, values)
    assert torch.equal(y, beta.to(dtype)[None].expand_as(y))
    n = ref.chain(cols)
    off = (n + 2) * U * values.double().abs()
    left = 3 * (n + 4) * U * off.square()
    assert bool((rstd.double() <= eps ** -0.5 * (1 + 4 * U)).all())
    assert bool((rstd.double() >= (eps + left) ** -0.5 * (1 - 4 * U)).all())


def corrected(x, gamma, beta, eps):
    """y, mean, rstd of float64 rows that vary less than their mean is, and bounds:
    the first mean is off by the roundings of its sum, the mean of the differences
    from it by those of theirs, the sum of the two is rounded once; and the squares'
    mean, var + off^2, and what is taken off it."""
    cols = x.shape[1]
    m = x.mean(1, keepdim=True)
    var = (x - m).square().mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    y = (x - m) * r * gamma + beta
    n = ref.chain(cols) + 4
    off = n * U * x.abs().mean(1, keepdim=True)
    dev = (x - m).abs().mean(1, keepdim=True) + off
    dmean = n * U * dev + U * m.abs()
    dvar = n * U * (var + off.square()) + 2 * off * n * U * dev + 4 * U * off.square()
    drel = 0.5 * dvar / (var + eps - dvar) + 4 * U
    dy = (gamma * r).abs() * (dmean + (x - m).abs() * (drel + 4 * U))
    dy = dy + 4 * U * (y.abs() + beta.abs()) + U * y.abs()
    return (y, m[:, 0], r[:, 0]), (dy, dmean[:, 0], (r * drel)[:, 0])


@pytest.mark.parametrize("center,spread", [(700.0, 2.0 ** -12), (1000.0, 1.0), (-40.0, 0.01)])
@pytest.mark.parametrize("cols", COLS)
def test_rows_that_hardly_vary(zpp, cols, center, spread):
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = center + spread * torch.randn(6, cols, device="cuda", generator=gen)
    gamma, beta = params(cols)
    got = forward(zpp, x, gamma, beta, 1e-12)
    want, bound = corrected(x.double(), gamma.double(), beta.double(), 1e-12)
    for g, w, b, what in zip(got, want, bound, ("y", "mean", "rstd")):
        ref.check(g, w, b, what)


@pytest.mark.parametrize("rows,cols", [(9000, 64), (4500, 1001), (1200, 4544), (700, 8201),
                                       (600, 20000)])
def test_rows_of_both_kinds(zpp, rows, cols):
    """Several rows one after the other in a workgroup, every third of which varies
    less than its mean is; each as if it were alone."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(rows, cols, device="cuda", generator=gen)
    far = torch.arange(rows, device="cuda") % 3 == 1
    x[far] += 500
    gamma, beta = params(cols)
    got = forward(zpp, x, gamma, beta, 1e-5)
    for part, form in ((far, corrected(x[far].double(), gamma.double(), beta.double(), 1e-5)),
                       (~far, ref.norm_forward(x[~far].double(), gamma.double(), beta.double(),
                                               1e-5, F32))):
        for g, w, b, what in zip(got, *form, ("y", "mean", "rstd")):
            ref.check(g[part], w, b, what)


@pytest.mark.parametrize("cols", COLS)
def test_variance_beyond_fp32(zpp, cols):
    """Squares that pass fp32: rstd is 0 and y the bias, no NaN, where the mean is 0
    and where it is far from 0."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(4, cols, device="cuda", generator=gen) * 2.0 ** 100
    x[1::2] += 2.0 ** 102
    gamma, beta = params(cols)
    y, mean, rstd = forward(zpp, x, gamma, beta, 1e-5)
    assert bool((rstd == 0).all()) and bool(torch.isfinite(mean).all())
    assert torch.equal(y, beta[None].expand_as(y))
