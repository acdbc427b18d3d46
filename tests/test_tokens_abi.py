"""The C ABI of the token operators on the CPU: bad arguments are rejected before any
HIP call, the binding's structures have the C compiler's layout, the kernels keep their
values in registers, and the host code (csrc/token_api.hip with counting stand-ins for its
launchers) is clean under AddressSanitizer and UndefinedBehaviorSanitizer.

Addresses are made up and never dereferenced: every call fails validation or is a
size-0 no-op without events.
"""
import ctypes
import os
import re
import subprocess

import pytest

import test_abi_sanitized as san
from paper_2407_01614_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
BF16, F32, I8 = 0, 1, 2
A = 0x7F0000000000
GB = 1 << 30


@pytest.fixture(scope="module")
def zpp():
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2407_01614_amd import zpp as mod
    return mod


def at(i, off=0):
    return A + i * GB + off


@pytest.mark.parametrize("mirror,name", [("Heads", "zpp_heads"), ("AdamTensor", "zpp_adam_tensor"),
                                         ("AdamTable", "zpp_adam_table")])
def test_layout(zpp, tmp_path, mirror, name):
    mirror = getattr(zpp, mirror)
    names = [f for f, _ in mirror._fields_]
    src = ('#include <stddef.h>\n#include <stdio.h>\n#include "zpp.h"\nint main(void){\n'
           '  printf("size %%zu\\n", sizeof(%s));\n  printf("top %%d\\n", ZPP_MAX_TOP);\n'
           '  printf("block %%d\\n", ZPP_ADAM_BLOCK);\n' % name
           + "".join('  printf("%s %%zu\\n", offsetof(%s, %s));\n' % (f, name, f) for f in names)
           + '  return 0;\n}\n')
    exe = str(tmp_path / "layout")
    r = subprocess.run(["gcc", "-x", "c", "-std=c99", "-D__HIP_PLATFORM_AMD__",
                        "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", "-",
                        "-o", exe], input=src, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = dict(line.split() for line in subprocess.run(
        [exe], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(got["size"]) == ctypes.sizeof(mirror)
    assert int(got["top"]) == zpp.MAX_TOP and int(got["block"]) == zpp.ADAM_BLOCK
    for f in names:
        assert int(got[f]) == getattr(mirror, f).offset, f


def turn(zpp, **kw):
    head = lambda i, off=0: bytes(zpp.Heads(at(i, off), 512, 0, 64, 1, 8))
    a = dict(x=head(0), out=head(1), k=None, k_out=None, type=BF16, tokens=10, dim=64, rotated=64,
             positions=at(2), turns=at(3), scale=1.0)
    a.update({k: head(*v) if isinstance(v, tuple) else v for k, v in kw.items()})
    found = {f(a["x"], a["out"], a["k"], a["k_out"], a["type"], a["tokens"], a["dim"],
               a["rotated"], a["positions"], a["turns"], 0, a["scale"], None, None, None)
             for f in (zpp.raw.zpp_rotary_forward, zpp.raw.zpp_rotary_backward)}
    assert len(found) == 1
    return found.pop()


def test_rotary_validation(zpp):
    assert turn(zpp, tokens=0) == zpp.ZPP_OK and turn(zpp, dim=0, rotated=0) == zpp.ZPP_OK
    for bad in (dict(x=None), dict(out=None), dict(k=(4,)), dict(k_out=(4,)), dict(type=I8),
                dict(type=-1), dict(rotated=63), dict(rotated=66), dict(dim=20000),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(positions=None),
                dict(turns=None), dict(tokens=0, rotated=63), dict(tokens=1 << 62)):
        assert turn(zpp, **bad) == zpp.ZPP_EINVAL, bad
    for bad in (dict(x=(0, 1)), dict(out=(1, 1)), dict(positions=at(2, 4)), dict(turns=at(3, 2)),
                dict(type=F32, x=(0, 2))):
        assert turn(zpp, **bad) == zpp.ZPP_EALIGN, bad
    for bad in (dict(out=(0, 2)), dict(k=(4,), k_out=(1,)), dict(k=(4,), k_out=(0,)),
                dict(k=(1,), k_out=(4,)), dict(out=(2,)), dict(out=(3,)), dict(positions=at(1, 1024))):
        assert turn(zpp, **bad) == zpp.ZPP_EOVERLAP, bad


R, V = 40, 1000


def mat(zpp, i, type=BF16, stride=V, off=0):
    return bytes(zpp.Matrix(None if i is None else at(i, off), None, stride, type))


def forward(zpp, **kw):
    a = dict(x=mat(zpp, 0), rows=R, vocab=V, targets=at(1), lp=at(2), lse=at(3), h=at(4), top=5,
             ids=at(5), tlp=at(6), ws=at(7))
    a.update(kw)
    a.setdefault("size", zpp.raw.zpp_log_probs_workspace(a["rows"], a["vocab"], a["top"]))
    return zpp.raw.zpp_log_probs_forward(a["x"], a["rows"], a["vocab"], a["targets"], a["lp"],
                                         a["lse"], a["h"], a["top"], a["ids"], a["tlp"], a["ws"],
                                         a["size"], None, None, None)


def test_log_probs_forward_validation(zpp):
    size = zpp.raw.zpp_log_probs_workspace
    need = size(R, V, 5)
    assert need >= R * 5 * 8 and size(R, V, 65) == 0 and size(R, 4, 5) == 0
    assert size(R, 1 << 31, 0) == 0 and size(1 << 62, V, 0) == 0 and size(R, 524289, 1) == 0
    assert size(1, 65024, 0) > 0 and size(8192, 65024, 0) == 0
    assert forward(zpp, rows=0) == zpp.ZPP_OK
    for bad in (dict(x=None), dict(x=mat(zpp, None)), dict(x=mat(zpp, 0, I8)), dict(targets=None),
                dict(lp=None), dict(ids=None), dict(tlp=None), dict(ws=None), dict(size=need - 1),
                dict(top=65), dict(vocab=4), dict(vocab=0, top=0), dict(vocab=1 << 31, top=0),
                dict(x=mat(zpp, 0, stride=V - 1)), dict(rows=0, top=65)):
        assert forward(zpp, **bad) == zpp.ZPP_EINVAL, bad
    for bad in (dict(x=mat(zpp, 0, off=1)), dict(targets=at(1, 4)), dict(lp=at(2, 2)),
                dict(ids=at(5, 1)), dict(ws=at(7, 8))):
        assert forward(zpp, **bad) == zpp.ZPP_EALIGN, bad
    for bad in (dict(lp=at(0)), dict(lse=at(2)), dict(h=at(1)), dict(ids=at(6)), dict(ws=at(0)),
                dict(tlp=at(7))):
        assert forward(zpp, **bad) == zpp.ZPP_EOVERLAP, bad


def backward(zpp, **kw):
    a = dict(x=mat(zpp, 0), rows=R, vocab=V, targets=at(1), lse=at(2), g=at(3), h=at(4), dh=at(5),
             dx=mat(zpp, 6))
    a.update(kw)
    return zpp.raw.zpp_log_probs_backward(a["x"], a["rows"], a["vocab"], a["targets"], a["lse"],
                                          a["g"], a["h"], a["dh"], a["dx"], None, None, None)


def train(zpp, **kw):
    a = dict(x=mat(zpp, 0, F32), rows=1, vocab=V, targets=at(1), lp=at(2), lse=at(3), h=at(4),
             g=at(5), dh=at(6), dx=mat(zpp, 7, F32), ws=at(8), size=GB)
    a.update(kw)
    return zpp.raw.zpp_log_probs_train(a["x"], a["rows"], a["vocab"], a["targets"], a["lp"],
                                       a["lse"], a["h"], a["g"], a["dh"], a["dx"], a["ws"],
                                       a["size"], None, None, None)


def test_log_probs_gradient_validation(zpp):
    assert backward(zpp, rows=0) == zpp.ZPP_OK and train(zpp, rows=0) == zpp.ZPP_OK
    for bad in (dict(x=None), dict(dx=None), dict(targets=None), dict(lse=None), dict(g=None),
                dict(h=None), dict(dh=None), dict(dx=mat(zpp, 6, F32)), dict(vocab=0),
                dict(x=mat(zpp, 0, I8), dx=mat(zpp, 6, I8))):
        assert backward(zpp, **bad) == zpp.ZPP_EINVAL, bad
    for bad in (dict(dx=mat(zpp, 0, off=2)), dict(dx=mat(zpp, 0, stride=V + 1)),
                dict(dx=mat(zpp, 3)), dict(lse=at(6))):
        assert backward(zpp, **bad) == zpp.ZPP_EOVERLAP, bad
    assert backward(zpp, g=at(3, 1)) == zpp.ZPP_EALIGN
    for bad in (dict(lse=None), dict(h=None), dict(g=None), dict(lp=None),
                dict(vocab=65024, ws=None, x=mat(zpp, 0, F32, 65024), dx=mat(zpp, 7, F32, 65024)),
                dict(vocab=65024, size=8, x=mat(zpp, 0, F32, 65024), dx=mat(zpp, 7, F32, 65024))):
        assert train(zpp, **bad) == zpp.ZPP_EINVAL, bad
    for bad in (dict(lp=at(0)), dict(dx=mat(zpp, 6, F32)), dict(lse=at(5)), dict(h=at(7, V))):
        assert train(zpp, **bad) == zpp.ZPP_EOVERLAP, bad


def table(zpp, tensors, state=F32, grad=F32, size=None):
    rows = (zpp.AdamTensor * len(tensors))(*[zpp.AdamTensor(*t) for t in tensors])
    need = zpp.raw.zpp_adam_tensors_table_bytes(len(tensors))
    host = ctypes.create_string_buffer(need + 16)
    where = ctypes.addressof(host)
    where += -where % 8
    found = zpp.AdamTable()
    st = zpp.raw.zpp_adam_tensors_table(rows, len(tensors), state, grad, where,
                                        need if size is None else size, ctypes.byref(found))
    return st, found


def tensor(i, n=1000, wd=0.1, **kw):
    a = dict(master=at(i), m=at(i, GB // 8), v=at(i, GB // 4), ms=at(i, GB // 2), vs=at(i, GB // 2 + GB // 8),
             g=at(i, 3 * GB // 4), out=at(i, 7 * GB // 8), n=n, wd=wd)
    a.update(kw)
    return tuple(a.values())


def test_adam_tensors_validation(zpp):
    st, found = table(zpp, [tensor(0), tensor(1, 0), tensor(2, 257)])
    assert st == zpp.ZPP_OK and (found.tiles, found.tensors) == (6, 2) and not found.table
    assert table(zpp, [])[0] == zpp.ZPP_OK
    for bad in (dict(master=None), dict(m=None), dict(v=None), dict(g=None), dict(wd=float("nan")),
                dict(n=1 << 63)):
        assert table(zpp, [tensor(0), tensor(1, **bad)])[0] == zpp.ZPP_EINVAL, bad
    assert table(zpp, [tensor(0, ms=None)], I8)[0] == zpp.ZPP_EINVAL
    assert table(zpp, [tensor(0, ms=None, vs=None, out=None)])[0] == zpp.ZPP_OK
    assert table(zpp, [tensor(0)], BF16)[0] == zpp.ZPP_EINVAL
    assert table(zpp, [tensor(0)], F32, I8)[0] == zpp.ZPP_EINVAL
    assert table(zpp, [tensor(0)], size=8)[0] == zpp.ZPP_EINVAL
    for bad in (dict(master=at(1, 2)), dict(m=at(1, GB // 8 + 1)), dict(g=at(1, 2)), dict(out=at(1, 1))):
        assert table(zpp, [tensor(1, **bad)])[0] == zpp.ZPP_EALIGN, bad
    assert table(zpp, [tensor(0, m=at(0, GB // 8 + 1), v=at(0, GB // 4 + 3))], I8)[0] == zpp.ZPP_OK
    for bad in (dict(master=at(0)), dict(m=at(0, 3996)), dict(out=at(0, GB // 4)),
                dict(g=at(0, 7 * GB // 8)), dict(v=at(1, GB // 8))):
        assert table(zpp, [tensor(0), tensor(1, **bad)])[0] == zpp.ZPP_EOVERLAP, bad
    assert table(zpp, [tensor(0), tensor(1, vs=at(0, GB // 2))], I8)[0] == zpp.ZPP_EOVERLAP
    assert table(zpp, [tensor(0), tensor(1, g=at(0, 3 * GB // 4))])[0] == zpp.ZPP_OK


def test_adam_tensors_step_validation(zpp):
    hp = lambda **kw: ctypes.byref(zpp.AdamHParams(*{**dict(
        lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, wd=0.0, adamw=1, step=1), **kw}.values()))
    none = zpp.AdamTable(None, 0, 0, F32, F32)
    step = lambda found, h=hp(): zpp.raw.zpp_adam_tensors_step(
        ctypes.byref(found) if found else None, h, None, None, None)
    assert step(none) == zpp.ZPP_OK
    for bad in (dict(wd=0.1), dict(step=0), dict(b1=1.0), dict(eps=-1.0), dict(lr=float("nan"))):
        assert step(none, hp(**bad)) == zpp.ZPP_EINVAL, bad
    assert step(None) == zpp.ZPP_EINVAL and step(none, None) == zpp.ZPP_EINVAL
    for bad in ((None, 5, 1, F32, F32), (at(0), 0, 1, F32, F32), (at(0), 5, 0, F32, F32),
                (at(0), 5, 1, BF16, F32), (at(0), 5, 1, F32, I8), (at(0), 1 << 32, 1, F32, F32)):
        assert step(zpp.AdamTable(*bad)) == zpp.ZPP_EINVAL, bad
    assert step(zpp.AdamTable(at(0, 8), 5, 1, F32, F32)) == zpp.ZPP_EALIGN


def test_adam_state_validation(zpp):
    save = lambda x=at(0), n=1000, m=1, c=at(1), s=at(2): zpp.raw.zpp_adam_state_save(
        x, n, m, c, s, None, None, None)
    load = lambda x=at(0), n=1000, m=1, c=at(1), s=at(2): zpp.raw.zpp_adam_state_load(
        c, s, n, m, x, None, None, None)
    for call in (save, load):
        assert call(n=0) == zpp.ZPP_OK
        for bad in (dict(x=None), dict(c=None), dict(s=None), dict(m=0), dict(m=3), dict(n=1 << 62)):
            assert call(**bad) == zpp.ZPP_EINVAL, bad
        assert call(x=at(0, 2)) == zpp.ZPP_EALIGN and call(s=at(2, 1)) == zpp.ZPP_EALIGN
        assert call(c=at(0, 8)) == zpp.ZPP_EOVERLAP and call(s=at(0)) == zpp.ZPP_EOVERLAP


@pytest.mark.skipif(not os.path.exists(build.hipcc()), reason="hipcc not found")
@pytest.mark.parametrize("source", ["rotary.hip", "log_probs.hip", "adam_tensors.hip"])
def test_no_kernel_spills(source, tmp_path):
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    r = subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-c",
                        "-Rpass-analysis=kernel-resource-usage", "-I", build.INCLUDE,
                        "-I", build.CSRC, os.path.join(build.CSRC, source),
                        "-o", str(tmp_path / "out.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    spills = re.findall(r"VGPRs Spill: (\d+)", r.stderr)
    scratch = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)
    assert names and len(names) == len(spills) == len(scratch)
    bad = [n for n, a, b in zip(names, spills, scratch) if int(a) or int(b)]
    assert not bad, bad


@pytest.mark.skipif(not san.have_toolchain(), reason="ROCm clang with sanitizer runtimes not found")
def test_token_abi_clean_under_sanitizers(tmp_path):
    inc = ["-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2407_01614_amd", "csrc"),
           "-I", os.path.join(san.ROCM, "include")]
    api, drv = str(tmp_path / "api.o"), str(tmp_path / "driver.o")
    exe = str(tmp_path / "token_abi_sanitized")
    for cmd in (
            [san.CLANGXX, "-x", "c++", "-std=c++17", *san.SAN, *inc, "-c",
             os.path.join(ROOT, "paper_2407_01614_amd", "csrc", "token_api.hip"), "-o", api],
            [san.CLANGXX, "-std=c++17", *san.SAN, *inc, "-c",
             os.path.join(HERE, "token_abi_sanitizer_driver.cpp"), "-o", drv],
            [san.CLANGXX, *san.SAN, api, drv, "-L", os.path.join(san.ROCM, "lib"), "-lamdhip64",
             "-Wl,-rpath," + os.path.join(san.ROCM, "lib"), "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, " ".join(cmd) + "\n" + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "sanitized token abi run ok" in r.stdout
