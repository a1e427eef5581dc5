"""Argument checks, plans and struct layouts of the loss and of the optimiser step at the C boundary and in the binding.  Runs
without a GPU: every call returns before touching the device."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2209_05433_b200 import api
from tests.test_abi import ROOT, _addresses

NULL, ENUM, SHAPE, ALIGN, UNSUPPORTED = 1, 2, 3, 4, 5


def test_cross_entropy_refusals():
    lib = api.load()
    one, odd = _addresses()
    d = api.CrossEntropyDesc(8, 64, 100, api.E4M3, api.E5M2, 64, 64)
    big = 1 << 40
    forward = lambda x=one, w=one, sx=one, sw=one, t=one, loss=one, lse=one, ws=one, n=big: lib.fp8_cross_entropy(  # noqa: E731
        ctypes.byref(d), x, w, sx, sw, t, loss, lse, ws, n, None)
    backward = lambda x=one, w=one, sx=one, sw=one, t=one, lse=one, g=one, dx=one, dxt=1, lddx=64, dw=one, dwt=1, lddw=64, ws=one, n=big: (  # noqa: E731
        lib.fp8_cross_entropy_backward(ctypes.byref(d), x, w, sx, sw, t, lse, g, dx, dxt, lddx, dw, dwt, lddw, ws, n, None))
    sizes = (ctypes.c_size_t(0), ctypes.c_size_t(0))
    size = lambda: lib.fp8_cross_entropy_workspace_bytes(ctypes.byref(d), ctypes.byref(sizes[0]), ctypes.byref(sizes[1]))  # noqa: E731
    assert size() == 0 and sizes[0].value > 0 and sizes[1].value >= 8 * 100
    assert lib.fp8_cross_entropy_workspace_bytes(None, None, None) == NULL
    for call in (forward, backward):
        for name in ("x", "w", "sx", "sw", "t", "lse", "ws"):
            assert call(**{name: None}) == NULL, name
        assert call(x=odd) == ALIGN and call(w=odd) == ALIGN and call(ws=odd) == ALIGN
        assert call(t=ctypes.c_void_p(20)) == ALIGN and call(lse=ctypes.c_void_p(18)) == ALIGN
        assert call(n=16) == SHAPE
    assert forward(loss=None) == NULL and backward(g=None) == NULL
    assert backward(dx=odd) == ALIGN and backward(dw=odd) == ALIGN and backward(lddx=63) == SHAPE and backward(lddw=60) == SHAPE
    assert backward(lddx=68) == ALIGN and backward(lddw=68, dwt=1) == ALIGN
    assert backward(dxt=2) == ENUM and backward(dwt=-1) == ENUM
    for field, bad, good, want in (("x_t", 3, 0, ENUM), ("w_t", -1, 1, ENUM), ("x_t", 2, 0, ENUM), ("tokens", -1, 8, SHAPE), ("width", 0, 64, SHAPE),
                                   ("vocab", 0, 100, SHAPE), ("ldx", 63, 64, SHAPE), ("ldw", 48, 64, SHAPE), ("ldx", 72, 64, ALIGN), ("ldw", 65, 64, ALIGN),
                                   ("tokens", 1 << 40, 8, UNSUPPORTED), ("vocab", 1 << 33, 100, UNSUPPORTED), ("width", 1 << 31, 64, UNSUPPORTED)):
        setattr(d, field, bad)
        assert forward() == want and backward() == want, field
        setattr(d, field, good)
    d.x_t = d.w_t = api.OPERAND_BF16
    d.ldx = 68
    assert forward(sx=None, sw=None) == ALIGN            # 136 bytes; the scales may be missing
    d.ldx, d.tokens = 64, 0
    assert forward(x=None, w=None, t=None, ws=None) == 0  # nothing to do, nothing touched
    assert backward(dw=None, x=None, ws=None) == 0


def test_workspaces_grow_with_the_work_but_hold_no_logits():
    for tokens, vocab in ((1, 128), (128, 131072), (4096, 65536), (65536, 131072)):
        forward, backward = api.load(), None
        forward, backward = ctypes.c_size_t(0), ctypes.c_size_t(0)
        d = api.CrossEntropyDesc(tokens, 4096, vocab, 0, 0, 4096, 4096)
        assert api.load().fp8_cross_entropy_workspace_bytes(ctypes.byref(d), ctypes.byref(forward), ctypes.byref(backward)) == 0
        assert forward.value <= tokens * (-(-vocab // 64) * 8 + 4 + 16)
        assert backward.value <= 4096 + max(tokens * 8192, 64 << 20) + 16 * 4096 * 4 * min(tokens, 256) + 4096 * 4 * tokens + 256 * tokens


def _items(n=3):
    items = (api.AdamWItem * n)()
    for i, it in enumerate(items):
        base = 1 << 20 << i
        it.g, it.p, it.m, it.v, it.n = base, 2 * base, 3 * base, 5 * base, (5, 0, 100000)[i % 3]
    return items


def test_adamw_plans_and_refusals():
    lib = api.load()
    one, odd = _addresses()
    items, sizes = _items(), api.AdamWSizes()
    size = lambda: lib.fp8_adamw_plan_size(items, 3, ctypes.byref(sizes))  # noqa: E731
    assert lib.fp8_adamw_plan_size(items, 3, None) == NULL and lib.fp8_adamw_plan_size(None, 3, ctypes.byref(sizes)) == NULL
    assert lib.fp8_adamw_plan_size(items, -1, ctypes.byref(sizes)) == SHAPE
    assert size() == 0 and sizes.count == 3 and sizes.chunk >= 2048 and sizes.chunk % 256 == 0 and sizes.amaxes == 0
    assert sizes.chunks == 1 + -(-100000 // sizes.chunk)
    table = (ctypes.c_uint8 * sizes.table_bytes)()
    assert lib.fp8_adamw_plan_fill(items, ctypes.byref(sizes), None) == NULL
    assert lib.fp8_adamw_plan_fill(items, ctypes.byref(sizes), table) == 0
    items[2].n = 1 << 24                                 # no longer the items the plan was sized for
    assert lib.fp8_adamw_plan_fill(items, ctypes.byref(sizes), table) == SHAPE
    items[2].n = 100000
    base = items[2].p
    for field, bad, good, want in (("g", 0, base, NULL), ("p", 0, base, NULL), ("m", 0, base, NULL), ("v", 0, base, NULL), ("p", base + 2, base, ALIGN),
                                   ("g", base + 1, base, ALIGN), ("m", base + 2, base, ALIGN), ("v", base + 1, base, ALIGN), ("n", -1, 100000, SHAPE),
                                   ("g_t", 2, 0, ENUM), ("p_t", -1, 0, ENUM), ("state", 2, 0, ENUM), ("state", 1, 0, NULL), ("weight_decay", -0.1, 0.0, UNSUPPORTED),
                                   ("weight_decay", float("nan"), 0.0, UNSUPPORTED), ("n", 1 << 60, 100000, UNSUPPORTED), ("copy_amax", 64, 0, NULL)):
        setattr(items[2], field, bad)
        assert size() == want, field
        setattr(items[2], field, good)
    items[2].copy, items[2].copy_t = base, 0             # a binary32 copy is no copy
    assert size() == ENUM
    items[2].copy_t = api.STORE_E4M3
    assert size() == NULL                                # codes need a scale
    items[2].copy_scale, items[2].copy_amax = 64, 128
    assert size() == 0 and sizes.amaxes == 1
    items[2].copy_scale = 66
    assert size() == ALIGN
    items[2].copy_scale = 64
    step = lambda ws=one, table=one, **o: lib.fp8_adamw_step(ctypes.byref(sizes), table, ws, ctypes.byref(api.AdamWOptions(  # noqa: E731
        **{**dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1), **o})), None)
    assert lib.fp8_adamw_step(None, one, one, ctypes.byref(api.AdamWOptions()), None) == NULL and lib.fp8_adamw_step(ctypes.byref(sizes), one, one, None, None) == NULL
    assert step(ws=None) == NULL and step(table=None) == NULL and step(ws=odd) == ALIGN and step(table=odd) == ALIGN
    nan = float("nan")
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=nan), dict(beta2=1.5), dict(eps=-1e-8), dict(eps=nan), dict(lr=nan), dict(lr=float("inf")), dict(step=0),
                dict(norm=64, max_norm=-1.0), dict(norm=64, max_norm=nan)):
        assert step(**bad) == UNSUPPORTED, bad
    assert step(norm=66) == ALIGN and step(lr_dev=65) == ALIGN and step(step_dev=68) == ALIGN
    none = api.AdamWSizes()
    assert lib.fp8_adamw_plan_size(items, 0, ctypes.byref(none)) == 0
    assert lib.fp8_adamw_step(ctypes.byref(none), None, one, ctypes.byref(api.AdamWOptions(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1)), None) == 0
    none.chunk = 0                                       # not a plan
    assert lib.fp8_adamw_step(ctypes.byref(none), None, one, ctypes.byref(api.AdamWOptions(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1)), None) == SHAPE


@pytest.mark.parametrize("sizes", [[1], [7, 77777], [16384, 4096] * 144, [1 << 26] * 4, [1234567, 333] * 18, [5000] * 1000, [0, 0]])
@pytest.mark.parametrize("state", [0, 1])
def test_adamw_chunks_cover_every_tensor_in_few_rounds(sizes, state):
    lib = api.load()
    items = (api.AdamWItem * len(sizes))()
    for it, n in zip(items, sizes):
        it.g = it.p = it.m = it.v = it.m_scale = it.v_scale = 4096
        it.n, it.state = n, state
    plan = api.AdamWSizes()
    assert lib.fp8_adamw_plan_size(items, len(sizes), ctypes.byref(plan)) == 0
    assert plan.chunk % 2048 == 0 and plan.chunks == sum(-(-n // plan.chunk) for n in sizes)
    table = (ctypes.c_uint8 * max(1, plan.table_bytes))()
    assert lib.fp8_adamw_plan_fill(items, ctypes.byref(plan), table) == 0
    owners = list((ctypes.c_int32 * plan.chunks).from_buffer(table, 128 * len(sizes))) if plan.chunks else []
    assert owners == [i for i, n in enumerate(sizes) for _ in range(-(-n // plan.chunk))]


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x, t, f = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    if torch.cuda.is_available():
        with pytest.raises(ValueError):
            api.fp8_cross_entropy(x, None, x, None, t, f, f)
    with pytest.raises(ValueError):
        api.AdamWPlan([f], [f], [f], [f, f])
    with pytest.raises(ValueError):
        api.AdamWPlan([f], [f], [f], [f])                # host tensors


def test_struct_layouts_match_the_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    fields = {"fp8_cross_entropy_desc": (api.CrossEntropyDesc, ["tokens", "width", "vocab", "x_t", "w_t", "ldx", "ldw"]),
              "fp8_adamw_item": (api.AdamWItem, ["g", "p", "m", "v", "m_scale", "v_scale", "copy", ("copy_scale_dev", "copy_scale"), ("copy_amax_dev", "copy_amax"),
                                                 "n", "weight_decay", "g_t", "p_t", "state", "copy_t"]),
              "fp8_adamw_plan": (api.AdamWSizes, ["count", "chunks", "chunk", "amaxes", "table_bytes", "workspace_bytes"]),
              "fp8_adamw_options": (api.AdamWOptions, ["lr", "beta1", "beta2", "eps", "step", "seed", ("norm_dev", "norm"), "lr_dev", "step_dev", "max_norm"])}
    lines, want = [], []
    for name, (cls, members) in fields.items():
        lines.append('printf("%%zu ", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for m in members:
            c, py = m if isinstance(m, tuple) else (m, m)
            lines.append('printf("%%zu ", offsetof(%s, %s));' % (name, c))
            want.append(getattr(cls, py).offset)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "fp8_b200.h"\nint main(void){%s return 0;}' % "".join(lines))
    exe = str(tmp_path / "layout")
    subprocess.run([gcc, "-I", os.path.join(ROOT, "include"), "-o", exe, str(src)], check=True)
    assert [int(v) for v in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()] == want
    # what the calls pass as bytes
    assert api._pack_cross_entropy(1, 2, 3, 1, 2, 6, 7) == bytes(api.CrossEntropyDesc(1, 2, 3, 1, 2, 6, 7))
    o = api.AdamWOptions(1e-3, 0.9, 0.99, 1e-8, 5, 6, 16, 32, 64, 2.0)
    assert api._pack_adamw(1e-3, 0.9, 0.99, 1e-8, 5, 6, 16, 32, 64, 2.0) == bytes(o)
    item = bytearray(ctypes.sizeof(api.AdamWItem))
    api._pack_adamw_item_into(item, 0, 16, 32, 48, 64, 80, 96, 112, 128, 144, 7, 0.5, 1, 0, 1, 3)
    want = api.AdamWItem(16, 32, 48, 64, 80, 96, 112, 128, 144, 7, 0.5, 1, 0, 1, 3)
    assert bytes(item) == bytes(want)
