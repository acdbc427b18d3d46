"""What the layer operators refuse, in the binding (type, device, shape, layout)
and in the library behind it (overlap, types that do not go together), and what
they take: each refusal raises before anything is enqueued."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
R, C = 6, 100


@pytest.fixture(scope="module")
def zpp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_01614_amd import zpp as mod
    return mod


def m(dtype=BF16, rows=R, cols=C):
    return torch.zeros(rows, cols, dtype=dtype, device="cuda")


def v(n, dtype=F32):
    return torch.zeros(n, dtype=dtype, device="cuda")


def ws(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def forward(zpp, **kw):
    a = dict(x=m(), gamma=v(C), beta=v(C), y=m(), mean=v(R), rstd=v(R), eps=1e-5)
    a.update(kw)
    zpp.layer_norm_forward(a.pop("x"), a.pop("gamma"), a.pop("beta"), a.pop("y"), a.pop("mean"),
                           a.pop("rstd"), **a)


def backward(zpp, **kw):
    a = dict(dy=m(), x=m(), gamma=v(C), mean=v(R), rstd=v(R), dx=m(), dgamma=v(C), dbeta=v(C),
             workspace=ws(zpp.layer_norm_backward_workspace(R, C)))
    a.update(kw)
    zpp.layer_norm_backward(*[a.pop(k) for k in ("dy", "x", "gamma", "mean", "rstd", "dx",
                                                 "dgamma", "dbeta", "workspace")], **a)


def grad(zpp, dy=None, x=None, dw=None, workspace=None, **kw):
    zpp.weight_grad(m() if dy is None else dy, m(cols=70) if x is None else x,
                    m(F32, C, 70) if dw is None else dw,
                    ws(zpp.weight_grad_workspace(R, C, 70)) if workspace is None else workspace,
                    **kw)


def test_binding_refuses(zpp):
    saved = zpp.empty_checkpoint(R, C)
    cases = [
        (TypeError, lambda: zpp.gelu_forward(m().half(), m())),
        (TypeError, lambda: zpp.gelu_forward(saved, m())),             # forward takes no checkpoint
        (TypeError, lambda: zpp.gelu_forward([1.0], m())),
        (TypeError, lambda: zpp.gelu_forward(m(), m(), saved=m())),
        (TypeError, lambda: zpp.gelu_backward(m(), saved[0], m())),    # codes without exponents
        (TypeError, lambda: zpp.gelu_backward(m(), saved + (1,), m())),
        (TypeError, lambda: zpp.checkpoint_load((saved[0], saved[1].int()), m())),
        (TypeError, lambda: zpp.checkpoint_load((saved[0].view(torch.uint8), saved[1]), m())),
        (ValueError, lambda: zpp.checkpoint_load((saved[0], saved[1][:3]), m())),
        (ValueError, lambda: zpp.gelu_forward(v(C), v(C))),            # not a matrix
        (ValueError, lambda: zpp.gelu_forward(m(), m(rows=R + 1))),
        (ValueError, lambda: zpp.gelu_forward(m().cpu(), m())),
        (ValueError, lambda: zpp.gelu_forward(m(cols=2 * C)[:, ::2], m())),
        (ValueError, lambda: zpp.gelu_forward(m(rows=C, cols=R).t(), m())),
        (TypeError, lambda: forward(zpp, gamma=v(C, torch.float16))),
        (TypeError, lambda: forward(zpp, beta=v(C, BF16))),            # not gamma's type
        (TypeError, lambda: forward(zpp, mean=v(R, torch.float64))),
        (ValueError, lambda: forward(zpp, gamma=v(C - 1))),
        (ValueError, lambda: forward(zpp, rstd=v(R - 1))),
        (ValueError, lambda: backward(zpp, dgamma=v(C - 1))),
        (ValueError, lambda: backward(zpp, workspace=ws(16))),
        (TypeError, lambda: backward(zpp, workspace=v(1 << 16))),
        (TypeError, lambda: backward(zpp, workspace=None)),
        (TypeError, lambda: grad(zpp, dy=m(F32))),
        (TypeError, lambda: grad(zpp, x=m(F32, cols=70))),
        (TypeError, lambda: grad(zpp, dw=m(BF16, C, 70))),
        (ValueError, lambda: grad(zpp, x=m(rows=R + 1, cols=70))),
        (ValueError, lambda: grad(zpp, dw=m(F32, C, 71))),
    ]
    for i, (kind, call) in enumerate(cases):
        with pytest.raises(kind):
            call()
            pytest.fail("case %d was taken" % i)
    torch.cuda.synchronize()


def refused(zpp, status, call):
    with pytest.raises(zpp.ZppError) as e:
        call()
    assert e.value.status == status


def test_library_refuses(zpp):
    x, wide = m(), m(cols=3 * C)
    refused(zpp, zpp.ZPP_EOVERLAP, lambda: zpp.gelu_forward(x, x))
    refused(zpp, zpp.ZPP_EOVERLAP, lambda: zpp.gelu_forward(wide[:, :C], wide[:, C - 1:2 * C - 1]))
    refused(zpp, zpp.ZPP_EOVERLAP, lambda: zpp.gelu_backward(m(), x, m(), a=x))
    refused(zpp, zpp.ZPP_EOVERLAP, lambda: backward(zpp, dx=x, y=x))
    refused(zpp, zpp.ZPP_EINVAL, lambda: zpp.gelu_forward(m(), m(F32)))
    refused(zpp, zpp.ZPP_EINVAL, lambda: zpp.gelu_forward(m()[:1].expand(R, C), m()))
    refused(zpp, zpp.ZPP_EINVAL, lambda: forward(zpp, residual=m()))
    refused(zpp, zpp.ZPP_EINVAL, lambda: forward(zpp, total=m()))
    refused(zpp, zpp.ZPP_EINVAL, lambda: forward(zpp, eps=-1.0))
    refused(zpp, zpp.ZPP_EINVAL, lambda: forward(zpp, eps=float("nan")))
    refused(zpp, zpp.ZPP_EINVAL, lambda: backward(zpp, x=m(F32)))
    torch.cuda.synchronize()


def test_column_ranges_of_one_matrix_are_apart(zpp):
    """Neighbouring column ranges as input and output: taken, and right."""
    wide = torch.randn(R, 3 * C, device="cuda").to(BF16)
    out = torch.empty(R, C, dtype=BF16, device="cuda")
    keep = wide.clone()
    zpp.gelu_forward(wide[:, C:2 * C], out)
    zpp.gelu_forward(wide[:, C:2 * C], wide[:, :C])
    assert torch.equal(wide[:, :C], out) and torch.equal(wide[:, C:], keep[:, C:])
    zpp.gelu_forward(wide[:, C:2 * C], wide[:, 2 * C:])
    assert torch.equal(wide[:, 2 * C:], out) and torch.equal(wide[:, C:2 * C], keep[:, C:2 * C])


def test_bits_of_bf16_are_taken(zpp):
    x = torch.randn(R, C, device="cuda").to(BF16)
    a, b = m(), m(torch.int16)
    zpp.gelu_forward(x, a)
    zpp.gelu_forward(x.view(torch.int16), b)
    assert torch.equal(a.view(torch.int16), b)
