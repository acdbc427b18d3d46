"""The C ABI of the layer operators on the CPU: bad arguments are rejected before
any HIP call, the binding's mirror of zpp_matrix has the C compiler's layout, and
the host code is clean under AddressSanitizer and UndefinedBehaviorSanitizer
(csrc/layer_api.hip with counting stand-ins for its launchers).

Addresses are made up and never dereferenced: every call fails validation or is a
size-0 no-op without events.
"""
import ctypes
import os
import subprocess

import pytest

import test_abi_sanitized as san

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
BF16, F32, I8 = 0, 1, 2
A = 0x7F0000000000
GB = 1 << 30


@pytest.fixture(scope="module")
def zpp():
    if not os.path.exists(os.path.join(ROOT, "paper_2407_01614_amd", "libzpp.so")):
        from paper_2407_01614_amd import build
        build.build()
    from paper_2407_01614_amd import zpp as mod
    return mod


def at(i, off=0):
    return A + i * GB + off


def test_matrix_layout(zpp, tmp_path):
    names = [f for f, _ in zpp.Matrix._fields_]
    src = ('#include <stddef.h>\n#include <stdio.h>\n#include "zpp.h"\nint main(void){\n'
           '  printf("size %zu\\n", sizeof(zpp_matrix));\n'
           + "".join('  printf("%s %%zu\\n", offsetof(zpp_matrix, %s));\n' % (f, f) for f in names)
           + '  printf("types %d\\n", ZPP_BF16 + 10 * ZPP_F32 + 100 * ZPP_I8);\n  return 0;\n}\n')
    exe = str(tmp_path / "layout")
    r = subprocess.run(["gcc", "-x", "c", "-std=c99", "-D__HIP_PLATFORM_AMD__",
                        "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", "-",
                        "-o", exe], input=src, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = dict(line.split() for line in subprocess.run(
        [exe], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(got["size"]) == ctypes.sizeof(zpp.Matrix)
    assert int(got["types"]) == 210
    for f in names:
        assert int(got[f]) == getattr(zpp.Matrix, f).offset, f


def mat(zpp, i, type=BF16, stride=1000, off=0, exps=None):
    if type == I8 and exps is None:
        exps = at(i, GB // 2)
    return bytes(zpp.Matrix(None if i is None else at(i, off), exps, stride, type))


R, C = 40, 1000


def test_checkpoint_validation(zpp):
    save = lambda x, s, rows=R, cols=C: zpp.raw.zpp_checkpoint_save(x, s, rows, cols, None, None,
                                                                    None)
    load = lambda s, o, rows=R, cols=C: zpp.raw.zpp_checkpoint_load(s, o, rows, cols, None, None,
                                                                    None)
    x, s = mat(zpp, 0), mat(zpp, 1, I8)
    for call, good in ((save, (x, s)), (load, (s, x))):
        for size in ((0, C), (R, 0), (0, 0)):
            assert call(*good, *size) == zpp.ZPP_OK
        assert call(None, good[1]) == zpp.ZPP_EINVAL
        assert call(good[0], None) == zpp.ZPP_EINVAL
        assert call(good[1], good[0]) == zpp.ZPP_EINVAL            # types the other way round
        assert call(*good, R, 1 << 31) == zpp.ZPP_EINVAL
        assert call(*good, 1 << 62, C) == zpp.ZPP_EINVAL
    assert save(mat(zpp, None), s) == zpp.ZPP_EINVAL
    assert save(x, bytes(zpp.Matrix(at(1), None, C, I8))) == zpp.ZPP_EINVAL
    assert save(mat(zpp, 0, stride=C - 1), s) == zpp.ZPP_EINVAL
    assert save(mat(zpp, 0, stride=1 << 62), s) == zpp.ZPP_EINVAL
    assert save(mat(zpp, 0, type=3), s) == zpp.ZPP_EINVAL
    assert save(mat(zpp, 0, type=-1), s) == zpp.ZPP_EINVAL
    assert save(mat(zpp, 0, off=1), s) == zpp.ZPP_EALIGN
    assert save(mat(zpp, 0, F32, off=2), s) == zpp.ZPP_EALIGN
    # bad sizes come before alignment, alignment before overlap
    assert save(mat(zpp, 0, off=1, stride=1), s) == zpp.ZPP_EINVAL
    assert save(mat(zpp, 1, off=1), s) == zpp.ZPP_EALIGN
    assert save(mat(zpp, 1), s) == zpp.ZPP_EOVERLAP
    # codes over exponents, and the last byte of the input
    assert save(x, mat(zpp, 1, I8, exps=at(1, R * C - 1))) == zpp.ZPP_EOVERLAP
    assert save(mat(zpp, 0), mat(zpp, 0, I8, off=2 * R * C - 1, exps=at(2))) == zpp.ZPP_EOVERLAP


def test_column_ranges(zpp):
    """Same distance between rows: ranges beside each other are apart, to the
    element; different distances are not looked into."""
    gelu = lambda u, a: zpp.raw.zpp_gelu_forward(u, R, 100, a, None, None, None, None)
    wide = lambda col, stride=300, type=BF16: mat(zpp, 0, type, stride, off=col * 2)
    assert gelu(wide(0), wide(99)) == zpp.ZPP_EOVERLAP
    assert gelu(wide(200), wide(101)) == zpp.ZPP_EOVERLAP
    assert gelu(wide(0), wide(300 - 99)) == zpp.ZPP_EOVERLAP     # reaches into the next row's
    assert gelu(wide(250), wide(49)) == zpp.ZPP_EOVERLAP         # over a row's end and into the next
    assert gelu(wide(0), wide(150, 301)) == zpp.ZPP_EOVERLAP
    assert gelu(wide(0), wide(0)) == zpp.ZPP_EOVERLAP
    assert gelu(wide(0), wide(300)) == zpp.ZPP_EOVERLAP          # the next row is the same place


def forward(zpp, **kw):
    a = dict(x=mat(zpp, 0), residual=None, gamma=at(1), beta=at(2), param=F32, rows=R, cols=C,
             eps=1e-5, y=mat(zpp, 3), total=None, saved=None, mean=at(4), rstd=at(5))
    a.update(kw)
    return zpp.raw.zpp_layer_norm_forward(
        a["x"], a["residual"], a["gamma"], a["beta"], a["param"], a["rows"], a["cols"], a["eps"],
        a["y"], a["total"], a["saved"], a["mean"], a["rstd"], None, None, None)


def test_norm_forward_validation(zpp):
    assert forward(zpp, rows=0) == zpp.ZPP_OK and forward(zpp, cols=0) == zpp.ZPP_OK
    E = zpp.ZPP_EINVAL
    for bad in (dict(x=None), dict(y=None), dict(gamma=None), dict(param=I8), dict(param=7),
                dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(residual=mat(zpp, 6)), dict(total=mat(zpp, 6)), dict(y=mat(zpp, 3, F32)),
                dict(x=mat(zpp, 0, I8)), dict(saved=mat(zpp, 6)), dict(cols=1 << 26),
                dict(residual=mat(zpp, 6, F32), total=mat(zpp, 7, F32)),
                dict(rows=0, eps=-1.0), dict(rows=0, x=None)):
        assert forward(zpp, **bad) == E, bad
    for bad in (dict(gamma=at(1, 2)), dict(beta=at(2, 1), param=BF16), dict(mean=at(4, 2)),
                dict(rstd=at(5, 1)), dict(x=mat(zpp, 0, off=1))):
        assert forward(zpp, **bad) == zpp.ZPP_EALIGN, bad
    for bad in (dict(y=mat(zpp, 0)), dict(mean=at(5)), dict(mean=at(0)), dict(rstd=at(1, 4 * C - 4)),
                dict(residual=mat(zpp, 6), total=mat(zpp, 6)),
                dict(residual=mat(zpp, 6), total=mat(zpp, 0)),
                dict(saved=mat(zpp, 3, I8)), dict(saved=mat(zpp, 6, I8, exps=at(4)))):
        assert forward(zpp, **bad) == zpp.ZPP_EOVERLAP, bad


def backward(zpp, **kw):
    need = zpp.raw.zpp_layer_norm_backward_workspace(kw.get("rows", R), kw.get("cols", C))
    a = dict(dy=mat(zpp, 0), x=mat(zpp, 1, I8), gamma=at(2), beta=at(3), param=BF16, mean=at(4),
             rstd=at(5), dres=mat(zpp, 6), rows=R, cols=C, dx=mat(zpp, 7), y=mat(zpp, 8),
             dgamma=at(9), dbeta=at(10), ws=at(11), size=need)
    a.update(kw)
    return zpp.raw.zpp_layer_norm_backward(
        a["dy"], a["x"], a["gamma"], a["beta"], a["param"], a["mean"], a["rstd"], a["dres"],
        a["rows"], a["cols"], a["dx"], a["y"], a["dgamma"], a["dbeta"], 1, a["ws"], a["size"],
        None, None, None)


def test_norm_backward_validation(zpp):
    need = zpp.raw.zpp_layer_norm_backward_workspace(R, C)
    assert need >= 8 * C
    assert zpp.raw.zpp_layer_norm_backward_workspace(0, C) == 0
    assert zpp.raw.zpp_layer_norm_backward_workspace(R, 1 << 26) == 0
    assert backward(zpp, rows=0) == zpp.ZPP_OK and backward(zpp, cols=0) == zpp.ZPP_OK
    for bad in (dict(dy=None), dict(x=None), dict(dx=None), dict(gamma=None), dict(mean=None),
                dict(rstd=None), dict(param=I8), dict(ws=None), dict(size=need - 1),
                dict(dx=mat(zpp, 7, F32)), dict(x=mat(zpp, 1, F32)), dict(dy=mat(zpp, 0, I8)),
                dict(y=mat(zpp, 8, I8)), dict(dres=mat(zpp, 6, F32)), dict(cols=1 << 26)):
        assert backward(zpp, **bad) == zpp.ZPP_EINVAL, bad
    for bad in (dict(ws=at(11, 8)), dict(dgamma=at(9, 2)), dict(dbeta=at(10, 1)),
                dict(mean=at(4, 2)), dict(gamma=at(2, 1))):
        assert backward(zpp, **bad) == zpp.ZPP_EALIGN, bad
    for bad in (dict(dx=mat(zpp, 0)), dict(y=mat(zpp, 7)), dict(dgamma=at(10)), dict(ws=at(0)),
                dict(dbeta=at(4)), dict(dx=mat(zpp, 6)), dict(ws=at(1, GB // 2)),
                dict(dgamma=at(2))):
        assert backward(zpp, **bad) == zpp.ZPP_EOVERLAP, bad


def test_gelu_validation(zpp):
    fwd = lambda u, a, s=None, rows=R: zpp.raw.zpp_gelu_forward(u, rows, C, a, s, None, None, None)
    bwd = lambda d, u, o, a=None, rows=R: zpp.raw.zpp_gelu_backward(d, u, rows, C, o, a, None, None,
                                                                   None)
    u, a, s = mat(zpp, 0), mat(zpp, 1), mat(zpp, 2, I8)
    assert fwd(u, a, s, 0) == zpp.ZPP_OK and bwd(u, s, a, None, 0) == zpp.ZPP_OK
    for bad in ((None, a), (u, None), (u, mat(zpp, 1, F32)), (s, a), (u, a, mat(zpp, 2))):
        assert fwd(*bad) == zpp.ZPP_EINVAL
    assert fwd(u, mat(zpp, 0)) == zpp.ZPP_EOVERLAP
    assert fwd(u, a, mat(zpp, 1, I8)) == zpp.ZPP_EOVERLAP
    for bad in ((None, s, a), (u, None, a), (u, s, None), (u, mat(zpp, 2, F32), a), (s, s, a),
                (u, s, a, mat(zpp, 3, F32))):
        assert bwd(*bad) == zpp.ZPP_EINVAL
    assert bwd(u, s, mat(zpp, 2)) == zpp.ZPP_EOVERLAP
    assert bwd(u, s, a, a) == zpp.ZPP_EOVERLAP


def grad(zpp, rows=100, n=300, k=200, **kw):
    a = dict(dy=mat(zpp, 0), x=mat(zpp, 1, I8), dw=mat(zpp, 2, F32), ws=at(4), size=GB)
    a.update(kw)
    return zpp.raw.zpp_weight_grad(a["dy"], a["x"], rows, n, k, a["dw"], 1, a["ws"], a["size"],
                                   None, None, None)


def test_weight_grad_validation(zpp):
    for size in (dict(rows=0), dict(n=0), dict(k=0)):
        assert grad(zpp, **size) == zpp.ZPP_OK, size   # accumulate: nothing to add
    for bad in (dict(dy=None), dict(x=None), dict(dw=None), dict(dy=mat(zpp, 0, F32)),
                dict(x=mat(zpp, 1, F32)), dict(dw=mat(zpp, 2, BF16)), dict(n=1 << 31),
                dict(rows=1 << 31), dict(k=1 << 31), dict(dy=mat(zpp, 0, stride=299)),
                dict(dw=mat(zpp, 2, F32, stride=199))):
        assert grad(zpp, **bad) == zpp.ZPP_EINVAL, bad
    assert grad(zpp, dw=mat(zpp, 2, F32, off=2)) == zpp.ZPP_EALIGN
    assert grad(zpp, dw=mat(zpp, 0, F32)) == zpp.ZPP_EOVERLAP
    assert grad(zpp, dw=mat(zpp, 1, F32, off=GB // 2)) == zpp.ZPP_EOVERLAP
    # the inputs may be one matrix
    assert grad(zpp, rows=0, x=mat(zpp, 0)) == zpp.ZPP_OK
    big = zpp.raw.zpp_weight_grad_workspace
    assert big(0, 5, 5) == 0 and big(5, 1 << 31, 5) == 0
    # sizes that split the tokens need their workspace
    for size in ((8192, 64, 64), (4096, 512, 512)):
        need = big(*size)
        if need:
            m = dict(rows=size[0], n=size[1], k=size[2])
            assert grad(zpp, ws=None, **m) == zpp.ZPP_EINVAL
            assert grad(zpp, size=need - 1, **m) == zpp.ZPP_EINVAL
            assert grad(zpp, ws=at(4, 8), **m) == zpp.ZPP_EALIGN
            assert grad(zpp, ws=at(1), **m) == zpp.ZPP_EOVERLAP


@pytest.mark.skipif(not san.have_toolchain(), reason="ROCm clang with sanitizer runtimes not found")
def test_layer_abi_clean_under_sanitizers(tmp_path):
    inc = ["-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2407_01614_amd", "csrc"),
           "-I", os.path.join(san.ROCM, "include")]
    api, drv = str(tmp_path / "api.o"), str(tmp_path / "driver.o")
    exe = str(tmp_path / "layer_abi_sanitized")
    for cmd in (
            [san.CLANGXX, "-x", "c++", "-std=c++17", *san.SAN, *inc, "-c",
             os.path.join(ROOT, "paper_2407_01614_amd", "csrc", "layer_api.hip"), "-o", api],
            [san.CLANGXX, "-std=c++17", *san.SAN, *inc, "-c",
             os.path.join(HERE, "layer_abi_sanitizer_driver.cpp"), "-o", drv],
            [san.CLANGXX, *san.SAN, api, drv, "-L", os.path.join(san.ROCM, "lib"), "-lamdhip64",
             "-Wl,-rpath," + os.path.join(san.ROCM, "lib"), "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, " ".join(cmd) + "\n" + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "sanitized layer abi run ok" in r.stdout
