"""The operators of include/qlinear_block.h on the CPU: the header's functions
are exported, its structures match the binding's, bad arguments are refused
before the GPU is touched (by the library and by the binding), and the rotary
frequencies are those of their formulas."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

import block_ref as R
from paper_2607_08526_amd import qlinear as ql

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "qlinear_block.h")
HIP_INCLUDE = "/opt/rocm/include"

OK, INVALID, SHAPE, ALIGN, RANGE, UNSUPPORTED, HIP = range(7)
MX, Q4, INT8, F16, F32, BF16 = 20, 4, 8, 16, 0, 1
# fake, never dereferenced device addresses
A16, A4, A2, A1 = 0x10000, 0x10004, 0x10002, 0x10001


@pytest.fixture(scope="module")
def lib():
    return ql.load()


def test_exports(lib):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(qlinear_\w+)\s*\(", src))
    assert len(names) == 7
    for n in names:
        assert hasattr(lib, n) and n in ql.EXPORTS


def test_structures(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None or not os.path.isdir(os.path.join(HIP_INCLUDE, "hip")):
        pytest.skip("no host C compiler or HIP headers")
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "qlinear_block.h"',
           'int main(void) {']
    pairs = (("ql_gated", ql._Gated), ("ql_gated_grad", ql._GatedGrad))
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


def test_sizes(lib):
    assert lib.qlinear_codes_bytes(MX, 6144, 2048) == 6144 * 1024
    assert lib.qlinear_mx_scales_bytes(6144, 2048) == 6144 * 64
    assert lib.qlinear_mx_scales_bytes(6144, 2047) == 0
    assert lib.qlinear_mx_scales_bytes(0, 64) == 0


def test_mx_format_errors(lib):
    """MXFP4 through the entry points of qlinear.h: their checks, scales at any byte."""
    f = lambda X=A16, xdt=BF16, M=4, K=64, c=A16, s=A1, N=16, Y=A16: lib.qlinear_forward(
        MX, X, xdt, M, K, c, s, N, Y, None)
    assert f(M=0) == OK
    assert f(K=48) == SHAPE and f(N=0) == SHAPE and f(M=-1) == SHAPE
    assert f(s=None) == INVALID and f(c=None) == INVALID and f(X=None) == INVALID
    assert f(xdt=2) == INVALID
    assert f(X=A2) == ALIGN and f(c=A2) == ALIGN and f(Y=A2) == ALIGN
    assert f(M=1 << 31) == UNSUPPORTED
    assert f(M=(1 << 31) - 1, N=(1 << 31) - 1) == UNSUPPORTED  # workgroups of a launch
    q = lambda W=A16, N=8, K=64, c=A16, s=A1: lib.qlinear_quantize(MX, W, N, K, c, s, None)
    assert q(K=40) == SHAPE and q(N=0) == SHAPE
    assert q(W=A4) == ALIGN and q(c=A4) == ALIGN and q(s=None) == INVALID
    ep = ql._Epilogue(None, 2, None, F32)  # SiLU is a gated pair's
    assert lib.qlinear_forward_ep(MX, A16, BF16, 4, 64, A16, A16, 16, A16, ctypes.byref(ep),
                                  None) == INVALID


def test_dequantize_errors(lib):
    d = lambda fmt=MX, c=A16, s=A2, N=4, K=64, W=A16, dt=F32: lib.qlinear_dequantize(
        fmt, c, s, N, K, W, dt, None)
    assert d(N=0) == OK
    assert d(fmt=F16) == INVALID and d(fmt=5) == INVALID and d(dt=2) == INVALID
    assert d(K=33) == SHAPE and d(K=0) == SHAPE and d(N=-1) == SHAPE
    assert d(N=1 << 35, K=32) == UNSUPPORTED and d(N=(1 << 63) - 1) == UNSUPPORTED
    assert d(c=None) == INVALID and d(s=None) == INVALID and d(W=None) == INVALID
    assert d(c=A4) == ALIGN and d(W=A4) == ALIGN and d(fmt=Q4, s=A1) == ALIGN


def test_mx_act_errors(lib):
    a = lambda X=A16, dt=BF16, M=4, K=64, q=A16, s=A1: lib.qlinear_mx_quantize_act(
        X, dt, M, K, q, s, None)
    assert a(M=0, X=None) == OK
    assert a(dt=3) == INVALID and a(K=16) == SHAPE and a(M=-1) == SHAPE and a(K=0) == SHAPE
    assert a(M=1 << 31) == UNSUPPORTED and a(M=1 << 20, K=1 << 20) == UNSUPPORTED
    assert a(X=None) == INVALID and a(q=None) == INVALID and a(s=None) == INVALID
    assert a(X=A4) == ALIGN and a(q=A4) == ALIGN
    f = lambda q=A16, s=A1, M=4, K=64, c=A16, w=A1, N=16, Y=A16, ep=None: lib.qlinear_mx_forward(
        q, s, M, K, c, w, N, Y, ep, None)
    assert f(M=0) == OK
    assert f(K=16) == SHAPE and f(N=0) == SHAPE and f(M=-1) == SHAPE
    assert f(M=1 << 31) == UNSUPPORTED and f(M=1 << 30, N=1 << 30) == UNSUPPORTED
    assert f(q=None) == INVALID and f(s=None) == INVALID and f(c=None) == INVALID
    assert f(w=None) == INVALID and f(Y=None) == INVALID
    assert f(q=A4) == ALIGN and f(c=A4) == ALIGN and f(Y=A2) == ALIGN
    assert f(ep=ctypes.byref(ql._Epilogue(None, 7, None, F32))) == INVALID
    assert f(ep=ctypes.byref(ql._Epilogue(A2, 0, None, F32))) == ALIGN


def gated(fmt=MX, X=A16, M=4, K=64, N=16, gc=A16, gs=A2, uc=A16, us=A2, bg=None, bu=None, act=2):
    return ql._Gated(fmt, X, M, K, N, gc, gs, uc, us, bg, bu, act)


def test_gated_errors(lib):
    f = lambda H=A16, dt=BF16, **kw: lib.qlinear_gated_forward(ctypes.byref(gated(**kw)), H, dt,
                                                               None)
    assert f(M=0, X=None, H=None) == OK
    assert lib.qlinear_gated_forward(None, A16, BF16, None) == INVALID
    for bad in (dict(fmt=F16), dict(fmt=7), dict(act=3), dict(act=-1), dict(dt=2), dict(gc=None),
                dict(gs=None), dict(uc=None), dict(us=None), dict(X=None), dict(H=None),
                dict(X=0x20000, H=0x20000)):
        assert f(**({"H": 0x30000} | bad)) == INVALID, bad
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(K=40)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(M=1 << 31), dict(N=1 << 31), dict(K=1 << 22),
                dict(M=1 << 30, N=1 << 30, H=0x30000)):
        assert f(**bad) == UNSUPPORTED, bad
    for bad in (dict(gc=A4), dict(uc=A4), dict(X=A4), dict(bg=A2), dict(bu=A1), dict(H=A1),
                dict(H=A2, dt=F32), dict(fmt=Q4, gs=A1), dict(fmt=INT8, us=A1)):
        assert f(**({"H": 0x30000} | bad)) == ALIGN, bad


def test_gated_backward_errors(lib):
    def f(dH=A16, dhdt=F32, dG=A16, dU=A16, dX=A16, dxdt=BF16, dWg=A16, dWu=A16, dwdt=F32,
          dbg=A4, dbu=A4, **kw):
        d = ql._GatedGrad(dH, dhdt, dG, dU, dX, dxdt, dWg, dWu, dwdt, dbg, dbu)
        return lib.qlinear_gated_backward(ctypes.byref(gated(**kw)), ctypes.byref(d), None)
    assert lib.qlinear_gated_backward(ctypes.byref(gated()), None, None) == INVALID
    assert f(M=0, dWg=None, dWu=None, dbg=None, dbu=None, dX=None, dH=None, dG=None,
             dU=None) == OK
    for bad in (dict(dhdt=2), dict(dxdt=2), dict(dwdt=2), dict(dWg=None), dict(dWu=None),
                dict(dH=None), dict(dG=None), dict(dU=None), dict(fmt=F16), dict(act=9)):
        assert f(**bad) == INVALID, bad
    # outputs that are an input, or each other
    p = lambda i: 0x100000 * i
    apart = dict(X=p(1), dH=p(2), dG=p(3), dU=p(4), dX=p(5), dWg=p(6), dWu=p(7), dbg=p(8),
                 dbu=p(9))
    for name, other in (("dG", "dH"), ("dU", "X"), ("dX", "X"), ("dU", "dG"), ("dWg", "dX"),
                        ("dWu", "dWg"), ("dbu", "dbg")):
        assert f(**(apart | {name: apart[other]})) == INVALID, (name, other)
    for bad in (dict(N=12), dict(K=40), dict(M=-1)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(M=1 << 22), dict(N=1 << 22), dict(M=1 << 21, N=1 << 21)):
        assert f(**bad) == UNSUPPORTED, bad
    for bad in (dict(dH=A2), dict(dH=A1, dhdt=BF16), dict(dG=A4), dict(dU=A4), dict(dX=A4),
                dict(dWg=A4), dict(dWu=A4), dict(dbg=A2), dict(dbu=A2)):
        assert f(**bad) == ALIGN, bad


def test_rotary_errors(lib):
    def f(x=A16, ldx=256, o=0x20000, ldo=256, dt=BF16, rows=4, heads=4, dh=64, rot=32, fr=A16,
          pos=A16, start=0, period=0):
        return lib.qlinear_rotary(x, ldx, o, ldo, dt, rows, heads, dh, rot, fr, pos, start, period,
                                  1.0, 0, 0, None)
    assert f(rows=0, x=None) == OK
    for bad in (dict(dt=2), dict(x=None), dict(o=None), dict(fr=None), dict(o=A16, ldo=300)):
        assert f(**bad) == INVALID, bad
    # elements of both x and o: the next element, the next row, half a row on
    for o, ldo in ((A16 + 2, 256), (A16 + 512, 256), (A16 + 256, 256), (A16 + 2046, 300)):
        assert f(x=A16, ldx=256, o=o, ldo=ldo) == INVALID, (o, ldo)
    assert f(x=A16 + 512, o=A16, ldx=512, ldo=512, heads=5) == INVALID
    for bad in (dict(rows=-1), dict(heads=0), dict(dh=0), dict(rot=0), dict(rot=7), dict(rot=66),
                dict(ldx=255), dict(ldo=255), dict(pos=None), dict(rot=-2)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(rows=1 << 24), dict(ldx=1 << 31), dict(heads=1 << 31)):
        assert f(**bad) == UNSUPPORTED, bad
    for bad in (dict(x=A1), dict(o=A1), dict(dt=F32, x=A2), dict(fr=A4), dict(pos=A4)):
        assert f(**bad) == ALIGN, bad


# ---- the binding: host tensors reach every check but the last -----------------------

def mx_weights(N=16, K=64):
    return torch.zeros((N, K // 2), dtype=torch.uint8), torch.zeros((N, K // 32), dtype=torch.uint8)


def bad_calls():
    c, s = mx_weights()
    X = torch.zeros((4, 64), dtype=torch.bfloat16)
    qx, sx = mx_weights(4)
    dH = torch.zeros((4, 16))
    f8, x = torch.zeros(16, dtype=torch.float64), torch.zeros((4, 256))
    gf, gb = ql.gated_forward, ql.gated_backward
    return [
        (TypeError, lambda: ql.forward(ql.FMT_MXFP4, X, c, s.to(torch.int16), 16)),
        (ValueError, lambda: ql.forward(ql.FMT_MXFP4, X, c, s[:, :1], 16)),
        (ValueError, lambda: ql.forward(ql.FMT_MXFP4, X, c, s, 16)),
        (ValueError, lambda: ql.quantize(ql.FMT_MXFP4, torch.zeros((4, 40)))),
        (ValueError, lambda: ql.dequantize(ql.FMT_F16, c, s)),
        (TypeError, lambda: ql.dequantize(ql.FMT_MXFP4, c.float(), s)),
        (ValueError, lambda: ql.dequantize(ql.FMT_MXFP4, c, s, out=torch.zeros((16, 32)))),
        (TypeError, lambda: ql.dequantize(ql.FMT_MXFP4, c, s, dtype=torch.float16)),
        (ValueError, lambda: ql.dequantize(ql.FMT_MXFP4, c, s)),
        (ValueError, lambda: ql.quantize_act_mx(torch.zeros((4, 40)))),
        (ValueError, lambda: ql.quantize_act_mx(torch.zeros((4, 0)))),
        (TypeError, lambda: ql.quantize_act_mx(torch.zeros((4, 64), dtype=torch.float64))),
        (ValueError, lambda: ql.quantize_act_mx(X, qx=torch.zeros((4, 64), dtype=torch.uint8))),
        (ValueError, lambda: ql.quantize_act_mx(X)),
        (ValueError, lambda: ql.forward_mx(qx, sx[:3], c, s, 16)),
        (ValueError, lambda: ql.forward_mx(qx, sx, c, s, 17)),
        (TypeError, lambda: ql.forward_mx(qx.float(), sx, c, s, 16)),
        (ValueError, lambda: ql.forward_mx(qx, sx, c, s, 16, bias=torch.zeros(15))),
        (ValueError, lambda: ql.forward_mx(qx, sx, c, s, 16)),
        (TypeError, lambda: gf(ql.FMT_MXFP4, X.float(), (c, s), (c, s))),
        (ValueError, lambda: gf(ql.FMT_F16, X, (c, s), (c, s))),
        (ValueError, lambda: gf(ql.FMT_MXFP4, X, (c, s), (c[:8], s))),
        (ValueError, lambda: gf(ql.FMT_Q4, X, (c, s.to(torch.int16)), (c, s[:3].to(torch.int16)))),
        (ValueError, lambda: gf(ql.FMT_MXFP4, X, (c, s), (c, s), bias=(None, torch.zeros(5)))),
        (ValueError, lambda: gf(ql.FMT_MXFP4, X, (c, s), (c, s), H=torch.zeros((4, 15)))),
        (TypeError, lambda: gf(ql.FMT_MXFP4, X, (c, s), (c, s), hdtype=torch.float16)),
        (ValueError, lambda: gf(ql.FMT_MXFP4, X, (c, s), (c, s))),
        (ValueError, lambda: gb(ql.FMT_MXFP4, X, (c, s), (c, s), dH[:3])),
        (TypeError, lambda: gb(ql.FMT_MXFP4, X, (c, s), (c, s), dH, dtype=torch.float16)),
        (ValueError, lambda: gb(ql.FMT_MXFP4, X, (c[:12], s[:12]), (c[:12], s[:12]),
                                dH[:, :12].contiguous())),
        (ValueError, lambda: gb(ql.FMT_MXFP4, X, (c, s), (c, s), dH)),
        (TypeError, lambda: ql.rotary(x, 4, f8.float())),
        (TypeError, lambda: ql.rotary(x.to(torch.float16), 4, f8)),
        (ValueError, lambda: ql.rotary(x, 5, f8)),
        (ValueError, lambda: ql.rotary(x, 8, f8, dh=16)),
        (ValueError, lambda: ql.rotary(x.t(), 1, f8)),
        (ValueError, lambda: ql.rotary(x, 0, f8)),
        (ValueError, lambda: ql.rotary(x, 4, f8[:0])),
        (TypeError, lambda: ql.rotary(x, 4, f8, positions=torch.zeros(4, dtype=torch.int32))),
        (ValueError, lambda: ql.rotary(x, 4, f8, positions=torch.zeros(3, dtype=torch.int64))),
        (TypeError, lambda: ql.rotary(x, 4, f8, out=x.to(torch.bfloat16))),
        (ValueError, lambda: ql.rotary(x, 4, f8, out=x[:3])),
        (ValueError, lambda: ql.rotary(x, 4, f8, T=0)),
        (ValueError, lambda: ql.rotary(x, 4, f8)),
    ]


@pytest.mark.parametrize("i", range(len(bad_calls())))
def test_binding_refuses(i):
    err, call = bad_calls()[i]
    with pytest.raises(err):
        call()


def test_rotary_frequencies():
    f, m = ql.rotary_frequencies(64, device="cpu")
    assert f.dtype == torch.float64 and m == 1.0
    for j in range(32):
        assert abs(f[j] - 10000.0 ** (-2 * j / 64)) <= 1e-15
    lin, _ = ql.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu")
    assert torch.allclose(lin, f / 4, rtol=1e-15)
    ntk, _ = ql.rotary_frequencies(64, scaling="ntk", factor=4.0, device="cpu")
    assert ntk[0] == 1.0 and abs(ntk[-1] / f[-1] - 0.25) < 1e-12
    y, m = ql.rotary_frequencies(64, scaling="yarn", factor=4.0, context=4096, device="cpu")
    assert abs(m - (0.1 * math.log(4.0) + 1)) < 1e-15
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(y[turns > 34], f[turns > 34])
    assert torch.allclose(y[turns < 0.7], f[turns < 0.7] / 4, rtol=1e-15)
    assert ((y <= f) & (y >= f / 4 * (1 - 1e-15))).all() and (y.diff() < 0).all()
    assert ql.rotary_frequencies(2, scaling="ntk", factor=2.0, device="cpu")[0].tolist() == [1.0]
    for bad in (dict(rot=3), dict(rot=0), dict(rot=64, scaling="other"), dict(rot=64, factor=0.5),
                dict(rot=64, base=1.0), dict(rot=64, scaling="yarn", factor=2.0)):
        with pytest.raises(ValueError):
            ql.rotary_frequencies(device="cpu", **bad)


def test_reference_quantizer():
    """block_ref's MXFP4 encoder against the rule in exact fractions."""
    import numpy as np
    from fractions import Fraction
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((40, 32)) * 2.0 ** rng.integers(-140, 120, (40, 1))).astype(np.float32)
    x[0] = 0
    x[1, :7] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    x[1, 7:] = 4.0
    codes, scales = R.mx_encode(x)
    mags = [Fraction(m) for m in R.MAGS]
    for r in range(40):
        v = [abs(Fraction(float(t))) for t in x[r]]
        e = -127
        if max(v):
            e = -200
            while Fraction(2) ** (e + 3) <= max(v):
                e += 1
            e = min(max(e, -127), 127)
        assert scales[r, 0] == e + 127
        for k in range(32):
            q = v[k] / Fraction(2) ** e
            best = min(range(8), key=lambda c: (abs(q - mags[c]), c % 2))
            assert codes[r, k] & 7 == best and codes[r, k] >> 3 == np.signbit(x[r, k])
