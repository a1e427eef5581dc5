"""Which workspaces the binding hands to its kernels, without a GPU: a stand-in for the library and for the capture state."""
import gc
import types
import weakref

import pytest
import torch

from paper_2209_05433_b200 import api

HEAD = 16384


@pytest.fixture
def state(monkeypatch):
    s = types.SimpleNamespace(capturing=False, stream=7)
    lib = types.SimpleNamespace(fp8_epilogue_backward_workspace_bytes=lambda M, N: HEAD + 4 * M * N,
                                fp8_quantize_current_workspace_bytes=lambda: 64)
    monkeypatch.setattr(api, "load", lambda: lib)
    monkeypatch.setattr(api, "_stream", lambda: s.stream)
    monkeypatch.setattr(api, "_scalar", lambda t, name: t.data_ptr())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: s.capturing)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for name in ("_workspaces", "_amax_workspaces", "_backward_workspaces"):
        monkeypatch.setattr(api, name, {})
    return s


CPU = torch.device("cpu")


def test_backward_workspace_is_kept_per_stream_and_grown(state):
    a = api.epilogue_backward_workspace(CPU, 8, 8)
    assert api.epilogue_backward_workspace(CPU, 4, 8) is a and a.numel() == HEAD + 256 and int(a.sum()) == 0
    state.stream = 8
    assert api.epilogue_backward_workspace(CPU, 8, 8) is not a
    state.stream = 7
    b = api.epilogue_backward_workspace(CPU, 8, 9)
    assert b is not a and api.epilogue_backward_workspace(CPU, 8, 8) is b


def test_a_capture_never_gets_a_kept_backward_workspace(state):
    """a kept buffer is freed when a larger one takes its place; a graph would go on writing to it"""
    kept = weakref.ref(api.epilogue_backward_workspace(CPU, 8, 8))
    state.capturing = True
    mine, other = api.epilogue_backward_workspace(CPU, 8, 8), api.epilogue_backward_workspace(CPU, 8, 8)
    assert len({mine.data_ptr(), other.data_ptr(), kept().data_ptr()}) == 3
    assert int(mine[:HEAD].sum()) == 0 and mine.numel() == HEAD + 256
    state.capturing = False
    api.epilogue_backward_workspace(CPU, 64, 64)
    gc.collect()
    assert kept() is None and len(api._backward_workspaces) == 1           # replaced, and nothing of the capture was kept


def test_a_capture_never_gets_a_kept_amax_workspace(state):
    amax = torch.zeros(1)
    ptr, kept, stream = api._amax_args(amax)
    assert ptr == amax.data_ptr() and kept is not None and stream == 7
    assert api._amax_args(amax) == (ptr, kept, 7)
    state.capturing = True
    assert api._amax_args(amax) == (ptr, None, 7) and api._amax_args(None) == (None, None, 7)
    state.capturing, state.stream = False, 9
    assert api._amax_args(amax)[1] not in (None, kept)


def test_a_current_scaling_workspace_made_inside_a_capture_is_not_kept(state):
    """its zeros are written by replays only, so a plain call could find it uncleared"""
    state.capturing = True
    mine = api.current_scaling_workspace(CPU)
    state.capturing = False
    kept = api.current_scaling_workspace(CPU)
    assert kept is not mine and api.current_scaling_workspace(CPU) is kept
    state.capturing = True
    assert api.current_scaling_workspace(CPU) is kept
