"""Argument checks and struct layouts of the fused operators at the C boundary.  Runs without a GPU: every call returns
before touching the device."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2209_05433_b200 import api
from tests.test_abi import ROOT, _addresses

NULL, ENUM, SHAPE, ALIGN, UNSUPPORTED = 1, 2, 3, 4, 5


def test_epilogue_refusals():
    lib = api.load()
    one, odd = _addresses()
    d = api.GemmDesc(64, 64, 64, 0, 0, 0, 0, 64, 64, 64, 1)
    e = api.Epilogue(api.ACT_SILU, api.STORE_BF16, api.SATURATE, api.BF16, api.BF16, api.BF16)
    call = lambda A=one, B=one, D=one, sa=one, sb=one, sd=one, ws=None: lib.fp8_gemm_epilogue(  # noqa: E731
        ctypes.byref(d), ctypes.byref(e), A, B, D, sa, sb, sd, None, ws, None)
    assert lib.fp8_gemm_epilogue(None, ctypes.byref(e), one, one, one, one, one, one, None, None, None) == NULL
    assert lib.fp8_gemm_epilogue(ctypes.byref(d), None, one, one, one, one, one, one, None, None, None) == NULL
    assert call(sa=None) == NULL and call(sb=None) == NULL and call(A=None) == NULL and call(D=None) == NULL
    assert call(ws=odd) == ALIGN
    assert call(A=odd) == ALIGN and call(B=odd) == ALIGN and call(D=odd) == ALIGN
    for name, bad, good in (("act", 5, 0), ("act", -1, 0), ("store", 4, 1), ("overflow", 2, 0), ("bias_t", 2, 1), ("residual_t", 7, 1), ("pre_t", -1, 1)):
        setattr(e, name, bad)
        assert call() == ENUM, name
        setattr(e, name, good)
    e.store = api.STORE_E4M3
    assert call(sd=None) == NULL                         # codes need a scale
    e.store = api.STORE_BF16
    e.residual, e.ldr = one, 63
    assert call() == SHAPE
    e.ldr = 68
    assert call() == ALIGN                               # 136 bytes
    e.residual, e.ldr = odd, 64
    assert call() == ALIGN
    e.residual, e.pre, e.ldp = None, one, 32
    assert call() == SHAPE
    e.pre, e.bias = None, ctypes.c_void_p(17)
    assert call() == ALIGN
    e.bias = None
    d.lda = 48
    assert call() == SHAPE
    d.lda, d.ldd = 64, 63
    assert call() == SHAPE
    d.ldd, d.K = 64, -1
    assert call() == SHAPE
    d.K, d.M, d.lda = 64, 1 << 31, 64
    assert call() == UNSUPPORTED
    d.M, d.acc = 64, 3
    assert call() == ENUM
    d.acc, d.M = 0, 0
    assert call(A=None, D=None) == 0                     # nothing to do, nothing touched


def test_gated_refusals():
    lib = api.load()
    one, odd = _addresses()
    d = api.GemmDesc(64, 64, 64, 0, 0, 0, 0, 64, 64, 64, 1)
    w = api.Gated(api.ACT_SILU, api.STORE_BF16, api.SATURATE, api.BF16)
    fwd = lambda Bu=one, H=one, sh=one: lib.fp8_gemm_gated(ctypes.byref(d), ctypes.byref(w), one, one, Bu, H, one, one, one, sh, None, None, None)  # noqa: E731
    bwd = lambda dU=one: lib.fp8_gemm_gated_backward(ctypes.byref(d), ctypes.byref(w), one, one, one, dU, one, one, one, None, None, None)  # noqa: E731
    assert fwd(Bu=None) == NULL and fwd(H=None) == NULL and fwd(Bu=odd) == ALIGN
    assert bwd() == NULL                                 # gate and up are read
    w.gate, w.ldg = one, 64
    assert fwd() == NULL                                 # both or neither
    w.up = one
    assert bwd(dU=None) == NULL and bwd(dU=odd) == ALIGN
    w.ldg = 60
    assert fwd() == SHAPE and bwd() == SHAPE
    w.ldg = 68
    assert fwd() == ALIGN and bwd() == ALIGN
    w.ldg, w.up = 64, odd
    assert fwd() == ALIGN
    w.up, w.gate_t = one, 3
    assert fwd() == ENUM and bwd() == ENUM
    w.gate_t, w.act = 1, 11
    assert fwd() == ENUM and bwd() == ENUM
    w.act, w.store = 4, api.STORE_E5M2
    assert fwd(sh=None) == NULL


def test_epilogue_backward_and_clip_refusals():
    lib = api.load()
    one, odd = _addresses()
    call = lambda M=8, N=64, act=4, dy=one, dt=1, ldy=64, pre=one, pt=1, ldp=64, store=1, ov=0, s=one, out=one, ldo=64, db=None, ws=None, wb=0: (  # noqa: E731
        lib.fp8_epilogue_backward(M, N, act, dy, dt, ldy, pre, pt, ldp, store, ov, s, out, ldo, db, None, ws, wb, None))
    assert call(act=5) == ENUM and call(dt=2) == ENUM and call(pt=-1) == ENUM and call(store=9) == ENUM and call(ov=2) == ENUM
    assert call(M=-1) == SHAPE and call(ldy=63) == SHAPE and call(ldp=8) == SHAPE and call(ldo=1) == SHAPE
    assert call(dy=None) == NULL and call(pre=None) == NULL and call(out=None) == NULL and call(store=2, s=None) == NULL
    assert call(dy=odd) == ALIGN and call(pre=odd) == ALIGN and call(out=odd) == ALIGN and call(ldy=68) == ALIGN
    need = lib.fp8_epilogue_backward_workspace_bytes(8, 64)
    assert call(db=one) == NULL and call(db=one, ws=one, wb=need - 1) == SHAPE and call(db=one, ws=odd, wb=need) == ALIGN
    assert call(M=0, dy=None, pre=None, out=None) == 0
    # plans are made on the host
    items = (api.ClipItem * 3)()
    sizes = api.ClipSizes()
    for i, n in enumerate((5, 0, 100000)):
        items[i].x, items[i].out, items[i].n = 4096 * (i + 1), 4096 * (i + 1), n
    assert lib.fp8_clip_plan_size(items, 3, None) == NULL and lib.fp8_clip_plan_size(None, 3, ctypes.byref(sizes)) == NULL
    assert lib.fp8_clip_plan_size(items, -1, ctypes.byref(sizes)) == SHAPE
    assert lib.fp8_clip_plan_size(items, 3, ctypes.byref(sizes)) == 0 and sizes.count == 3 and sizes.chunks == 1 + 0 + 4
    table = (ctypes.c_uint8 * sizes.table_bytes)()
    assert lib.fp8_clip_plan_fill(items, ctypes.byref(sizes), None) == NULL
    assert lib.fp8_clip_plan_fill(items, ctypes.byref(sizes), table) == 0
    items[2].n = 1 << 20                                 # no longer the items the plan was sized for
    assert lib.fp8_clip_plan_fill(items, ctypes.byref(sizes), table) == SHAPE
    items[2].n, items[2].x = 100000, 4098
    assert lib.fp8_clip_plan_size(items, 3, ctypes.byref(sizes)) == ALIGN
    items[2].x, items[2].x_t = 12288, 4
    assert lib.fp8_clip_plan_size(items, 3, ctypes.byref(sizes)) == ENUM
    items[2].x_t, items[2].out_t = 0, 1                  # in place keeps its type
    assert lib.fp8_clip_plan_size(items, 3, ctypes.byref(sizes)) == ENUM
    items[2].out_t, items[2].n = 0, -2
    assert lib.fp8_clip_plan_size(items, 3, ctypes.byref(sizes)) == SHAPE
    for bad in (-1.0, float("nan")):
        assert lib.fp8_grad_clip(ctypes.byref(sizes), one, one, bad, one, None) == UNSUPPORTED
    assert lib.fp8_grad_norm(ctypes.byref(sizes), None, one, one, None) == NULL
    assert lib.fp8_grad_norm(ctypes.byref(sizes), one, one, None, None) == NULL
    assert lib.fp8_grad_norm(ctypes.byref(sizes), odd, one, one, None) == ALIGN


def test_struct_layouts_match_the_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    fields = {"fp8_epilogue": (api.Epilogue, ["act", "store", "overflow", "bias_t", "residual_t", "pre_t", ("scale_inv_b_vec_dev", "scale_inv_b_vec"), "bias",
                                              "residual", "pre", "ldr", "ldp"]),
              "fp8_gated": (api.Gated, ["act", "store", "overflow", "gate_t", "gate", "up", "ldg"]),
              "fp8_clip_item": (api.ClipItem, ["x", "out", "n", "x_t", "out_t"]),
              "fp8_clip_plan": (api.ClipSizes, ["count", "chunks", "table_bytes", "workspace_bytes"])}
    lines, want = [], []
    for name, (cls, members) in fields.items():
        lines.append('printf("%%zu ", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for m in members:
            c, py = m if isinstance(m, tuple) else (m, m)
            lines.append('printf("%%zu ", offsetof(%s, %s));' % (name, c))
            want.append(getattr(cls, py).offset)
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "fp8_b200.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.check_call([gcc, "-std=c11", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == want
