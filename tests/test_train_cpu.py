"""The operators of include/qlinear_train.h on the CPU: the header's functions are
exported, its structures match the binding's, and bad arguments are refused before the
GPU is touched (by the library and by the binding)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2607_08526_amd import qlinear as ql

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "qlinear_train.h")
HIP_INCLUDE = "/opt/rocm/include"

OK, INVALID, SHAPE, ALIGN, RANGE, UNSUPPORTED, HIP = range(7)
F32, BF16 = 0, 1
# fake, never dereferenced device addresses, far apart
A, B, C, D, E, F = (0x1000000 * k for k in range(1, 7))


@pytest.fixture(scope="module")
def lib():
    return ql.load()


def test_exports(lib):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(qlinear_\w+)\s*\(", src))
    assert len(names) >= 2
    for n in names:
        assert hasattr(lib, n) and n in ql.EXPORTS


def test_structures(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None or not os.path.isdir(os.path.join(HIP_INCLUDE, "hip")):
        pytest.skip("no host C compiler or HIP headers")
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "qlinear_train.h"',
           'int main(void) {']
    pairs = [("ql_norm", ql._Norm), ("ql_norm_grad", ql._NormGrad)]
    for name, cls in pairs:
        src.append(f'printf("%zu\\n", sizeof({name}));')
        src += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    c, exe = tmp_path / "l.c", tmp_path / "l"
    c.write_text("\n".join(src + ["return 0; }"]))
    subprocess.run([cc, "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    HIP_INCLUDE, str(c), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    want = []
    for _, cls in pairs:
        want += [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert [int(v) for v in out] == want


def norm(lib, **kw):
    n = dict(x=A, ldx=64, xdt=BF16, res=B, ldr=64, rdt=F32, weight=C, eps=1e-6, M=4, N=64, h=D,
             ldh=64, y=E, ldy=64, ydt=BF16, qx=None, sx=None)
    n.update(kw)
    return lib.qlinear_rms_norm(ctypes.byref(ql._Norm(**n)), None)


def test_norm_errors(lib):
    assert lib.qlinear_rms_norm(None, None) == INVALID
    assert norm(lib, M=0) == OK and norm(lib, M=0, x=None, h=None, y=None) == OK
    assert norm(lib, M=-1) == SHAPE and norm(lib, N=0) == SHAPE
    for ld in ("ldx", "ldr", "ldh", "ldy"):
        assert norm(lib, **{ld: 63}) == SHAPE and norm(lib, **{ld: 1 << 31}) == UNSUPPORTED
    assert norm(lib, N=16385, ldx=20000, ldr=20000, ldh=20000, ldy=20000) == UNSUPPORTED
    assert norm(lib, M=1 << 24) == UNSUPPORTED
    for dt in ("xdt", "rdt", "ydt"):
        assert norm(lib, **{dt: 2}) == INVALID
    assert norm(lib, x=None) == INVALID and norm(lib, h=None, y=None) == INVALID
    for eps in (-1e-9, float("nan"), float("inf")):
        assert norm(lib, eps=eps) == INVALID
    assert norm(lib, qx=F) == INVALID and norm(lib, sx=F) == INVALID
    big = dict(ldx=96, ldr=96, ldh=96, ldy=96, qx=F, sx=F + 4096)
    assert norm(lib, N=72, **big) == SHAPE  # no whole blocks
    assert norm(lib, N=96, **{**big, "qx": F + 8}) == ALIGN
    assert norm(lib, N=96, **{**big, "sx": F + 4097}) == ALIGN
    assert norm(lib, x=A + 1) == ALIGN and norm(lib, res=B + 2) == ALIGN
    assert norm(lib, h=D + 2) == ALIGN and norm(lib, y=E + 1) == ALIGN
    assert norm(lib, weight=C + 2) == ALIGN


def test_norm_aliases(lib):
    """In place is the same rows one by one; anything else that shares elements is
    refused (M == 0 would pass the last check, so these stop before a launch)."""
    assert norm(lib, h=B + 4) == INVALID                    # shifted
    assert norm(lib, h=B, ldh=72) == INVALID                # another stride
    assert norm(lib, y=B) == INVALID                        # bf16 over fp32
    assert norm(lib, y=E, h=E) == INVALID and norm(lib, y=D + 64 * 4 * 3) == INVALID
    assert norm(lib, weight=D) == INVALID
    assert norm(lib, y=C) == INVALID
    assert norm(lib, qx=A, sx=F) == INVALID and norm(lib, qx=F, sx=F + 16) == INVALID
    assert norm(lib, h=B + 128, ldr=96, ldh=96) == INVALID  # columns that overlap
    assert norm(lib, qx=F, sx=E) == INVALID


def grad(lib, **kw):
    g = dict(dy=A, lddy=64, dydt=BF16, h=B, ldh=64, hdt=F32, dres=C, lddres=64, weight=D, eps=1e-6,
             M=4, N=64, dx=E, lddx=64, dxdt=F32, dw=F)
    g.update(kw)
    return lib.qlinear_rms_norm_backward(ctypes.byref(ql._NormGrad(**g)), None)


def test_norm_backward_errors(lib):
    assert lib.qlinear_rms_norm_backward(None, None) == INVALID
    assert grad(lib, M=0, dw=None) == OK
    assert grad(lib, M=-1) == SHAPE and grad(lib, N=0) == SHAPE
    for ld in ("lddy", "ldh", "lddres", "lddx"):
        assert grad(lib, **{ld: 63}) == SHAPE and grad(lib, **{ld: 1 << 31}) == UNSUPPORTED
    assert grad(lib, N=16385, lddy=20000, ldh=20000, lddres=20000, lddx=20000) == UNSUPPORTED
    assert grad(lib, M=1 << 24) == UNSUPPORTED
    for dt in ("dydt", "hdt", "dxdt"):
        assert grad(lib, **{dt: 5}) == INVALID
    for p in ("dy", "h", "dx"):
        assert grad(lib, **{p: None}) == INVALID
    assert grad(lib, eps=-1.0) == INVALID
    assert grad(lib, dy=A + 1) == ALIGN and grad(lib, h=B + 2) == ALIGN
    assert grad(lib, dx=E + 2) == ALIGN and grad(lib, dw=F + 2) == ALIGN
    assert grad(lib, dres=C + 1) == ALIGN and grad(lib, weight=D + 1) == ALIGN
    assert grad(lib, dx=A) == INVALID                       # fp32 over bf16
    assert grad(lib, dx=B + 4) == INVALID and grad(lib, dx=C, lddx=96) == INVALID
    assert grad(lib, dw=D) == INVALID and grad(lib, dw=E) == INVALID
    assert grad(lib, dw=B + 64 * 4 * 3) == INVALID


def test_binding_refuses_norm():
    x = torch.zeros((4, 64))
    with pytest.raises(ValueError, match="device"):
        ql.rms_norm(x)
    with pytest.raises(TypeError, match="dtype"):
        ql.rms_norm(x.half())
    with pytest.raises(ValueError, match="2-D"):
        ql.rms_norm(x[0])
    with pytest.raises(ValueError, match="stride"):
        ql.rms_norm(x.t())
    with pytest.raises(ValueError, match="shape"):
        ql.rms_norm(x, torch.ones(63))
    with pytest.raises(TypeError, match="dtype"):
        ql.rms_norm(x, torch.ones(64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="eps"):
        ql.rms_norm(x, eps=-1.0)
    with pytest.raises(ValueError, match="shape"):
        ql.rms_norm(x, residual=x[:3])
    with pytest.raises(TypeError, match="dtype"):
        ql.rms_norm(x, residual=x, h=x.to(torch.bfloat16))
    with pytest.raises(ValueError, match="multiple"):
        ql.rms_norm_int8(x[:, :40])
    with pytest.raises(TypeError, match="dtype"):
        ql.rms_norm_int8(x, qx=torch.zeros((4, 64), dtype=torch.uint8))
    with pytest.raises(TypeError, match="dtype"):
        ql.rms_norm_backward(x, x, dres=x.to(torch.bfloat16))
    with pytest.raises(ValueError, match="at least 64 columns"):
        ql.rms_norm_backward(x[:, :63], x)
    with pytest.raises(ValueError, match="device"):
        ql.rms_norm_backward(x, x)
