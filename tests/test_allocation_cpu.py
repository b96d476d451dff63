"""How outputs are allocated where torch's shortest way, which is not public, is another one or gone.  No CUDA call."""
import sys
import types

import pytest
import torch


def _allocations(monkeypatch, short):
    """What torch.empty_strided is asked for when an output is made and `short` is all there is of the shortest way."""
    from paper_2605_09681_gb300 import _fast_calls
    guards = types.ModuleType("torch._C._dynamo.guards")
    if short is not None:
        guards._empty_strided_cuda = short
    monkeypatch.setitem(sys.modules, "torch._C._dynamo.guards", guards)
    asked = []
    monkeypatch.setattr(torch, "empty_strided", lambda *a, **kw: asked.append((a, kw)) or "plain")
    new, _, _ = _fast_calls()
    return new((4, 2, 64), (128, 64, 1), torch.bfloat16), asked


@pytest.mark.parametrize("short", [None, lambda shape: "other", lambda shape, strides, dtype, device: "other"])
def test_without_it(monkeypatch, short):
    out, asked = _allocations(monkeypatch, short)
    assert out == "plain"
    assert asked == [(((4, 2, 64), (128, 64, 1)), dict(dtype=torch.bfloat16, device="cuda"))]


def test_with_it(monkeypatch):
    out, asked = _allocations(monkeypatch, lambda shape, strides, dtype: (shape, strides, dtype))
    assert out == ((4, 2, 64), (128, 64, 1), torch.bfloat16) and not asked


def test_what_runs_out_is_not_asked_for_again(monkeypatch):
    """Errors of the allocation itself (no memory) are the caller's."""
    def short(shape, strides, dtype):
        raise RuntimeError("out of memory")
    with pytest.raises(RuntimeError, match="out of memory"):
        _allocations(monkeypatch, short)
