"""Layer norm's backward pass where a row's lanes hold more than the row: what a
lane has in place of elements past the row's end, or of another lane's, reaches no
sum, also where a number made of it would pass fp32."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def zpp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_01614_amd import zpp as mod
    return mod


def backward(zpp, dy, x, gamma, beta, mean, rstd, again):
    rows, cols = dy.shape
    dx = torch.empty_like(dy)
    y = torch.empty_like(dy) if again else None
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(zpp.layer_norm_backward_workspace(rows, cols), dtype=torch.uint8,
                     device="cuda")
    zpp.layer_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db, ws,
                            beta=beta if again else None, y=y)
    return dx, dg, db, y


def compare(got, dy, x, gamma, beta, mean, rstd, dtype):
    want, bound = ref.norm_backward(dy.double(), x, gamma.double(), beta.double(), mean.double(),
                                    rstd.double(), None, dtype)
    for g, w, b, what in zip(got, want, bound, ("dx", "dgamma", "dbeta", "y")):
        if g is not None:
            ref.check(g, w, b, what)


@pytest.mark.parametrize("again", [False, True], ids=["", "y"])
@pytest.mark.parametrize("from_saved", [False, True], ids=["plain", "i8"])
@TYPES
@pytest.mark.parametrize("cols", [5, 64, 72, 100, 520, 1001, 4544, 8200, 8201, 12000, 16390])
def test_large_rows_of_one_value(zpp, cols, dtype, from_saved, again):
    """A mean of 2^110 and an rstd of 2^20, as a row of that value has them: their
    product passes fp32, the row's own elements are 0."""
    rows = 3
    x = torch.full((rows, cols), 2.0 ** 110, device="cuda").to(dtype)
    x[1] = -x[1]
    mean, rstd = x[:, 0].float().contiguous(), torch.full((rows,), 2.0 ** 20, device="cuda")
    dy = ref.values(rows, cols, cols, dtype, std=1e-3)
    gamma = ref.values(1, cols, 1, F32)[0]
    beta = ref.values(1, cols, 2, F32)[0]
    arg = ref.saved(x)[0] if from_saved else x
    got = backward(zpp, dy, arg, gamma, beta, mean, rstd, again)
    compare(got, dy, x.double(), gamma, beta, mean, rstd, dtype)


@TYPES
@pytest.mark.parametrize("cols", [69, 1025, 4545, 8193, 8257])
def test_last_elements_of_another_block(zpp, cols, dtype):
    """The lane of a row's last, partial chunk also loads elements of the block
    before, whose codes with the last block's exponent, the largest there is, pass
    fp32."""
    rows = 3
    x = ref.values(rows, cols, cols, dtype)
    x[:, :cols // 64 * 64] *= 10
    last = cols // 64 * 64
    x[:, last - 8:last] = 127.0
    x[:, last:] = 3.389e38
    x[1, last:] = -3.389e38
    mean = torch.zeros(rows, device="cuda")
    rstd = torch.full((rows,), 2.0 ** -110, device="cuda")
    arg, values = ref.saved(x)
    assert int(arg[1][0, -1]) == 249
    dy = ref.values(rows, cols, cols + 1, dtype, std=1e-3)
    gamma, beta = ref.values(1, cols, 1, F32)[0], ref.values(1, cols, 2, F32)[0]
    for again in (False, True):
        got = backward(zpp, dy, arg, gamma, beta, mean, rstd, again)
        compare(got, dy, values, gamma, beta, mean, rstd, dtype)
