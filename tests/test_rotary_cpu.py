"""Host-side checks of the rotary positions' C ABI.  No kernel runs."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2605_09681_gb300 import build, _lib
    build.build()
    return _lib.load()


def _cfg(**kw):
    from paper_2605_09681_gb300._lib import FkRotaryConfig
    base = dict(head_dim=128, dim=128, style=0, n_axes=1, pairs=(64, 0, 0, 0), scaling=0, original_tokens=4096, base=1e4,
                factor=4.0, slow_turns=1.0, fast_turns=32.0, magnitude=0.0, frequencies=None)
    base.update(kw)
    base["pairs"] = (ctypes.c_int32 * 4)(*base["pairs"])
    if base["frequencies"] is not None:
        base["frequencies"] = (ctypes.c_double * len(base["frequencies"]))(*base["frequencies"])
    return FkRotaryConfig(*base.values())


def _make(lib, **kw):
    from paper_2605_09681_gb300._lib import FkRotary
    c, r = _cfg(**kw), FkRotary()
    return lib.fk_rotary_make(ctypes.byref(c), ctypes.byref(r)), r


def test_struct_layouts():
    from paper_2605_09681_gb300._lib import FkRotary, FkRotaryConfig
    assert ctypes.sizeof(FkRotaryConfig) == 88 and FkRotaryConfig.base.offset == 40
    assert ctypes.sizeof(FkRotary) == 1024 + 4 + 16 + 16 + 4


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "ramp"])
@pytest.mark.parametrize("pairs", [(64,), (22, 21, 21), (30, 2, 2, 30)])
def test_turns_are_the_frequencies(lib, scaling, pairs):
    """A double has 53 bits, pow at most one step off, and the fraction 64: 2^-51 of a frequency together with the
    scalings' few roundings, and 2^-64."""
    from oracle import linear_state as R
    code = {"none": 0, "linear": 1, "base": 2, "ramp": 3}[scaling]
    st, r = _make(lib, n_axes=len(pairs), pairs=pairs + (0,) * (4 - len(pairs)), scaling=code)
    assert st == 0
    freq, m = R.frequencies(pairs, 1e4, scaling, 4.0, 4096)
    got = np.array(list(r.turns)[:64], dtype=np.float64) * 2.0 ** -64 * 2 * np.pi
    assert (np.abs(got - freq) <= 2.0 ** -48 * np.array(freq) + 2 * np.pi * 2.0 ** -64).all()
    assert abs(r.magnitude - m) <= 2.0 ** -23 and list(r.first)[: len(pairs)] == [sum(pairs[:i]) for i in range(len(pairs))]


@pytest.mark.parametrize("bad", [
    dict(head_dim=120 + 4), dict(head_dim=264, dim=264, pairs=(132, 0, 0, 0)), dict(dim=0, pairs=(0, 0, 0, 0)), dict(dim=136, pairs=(68, 0, 0, 0)),
    dict(dim=120, pairs=(60, 0, 0, 0)), dict(pairs=(63, 0, 0, 0)), dict(style=2), dict(style=-1), dict(n_axes=0), dict(n_axes=5),
    dict(n_axes=2, pairs=(64, 0, 0, 0)), dict(n_axes=2, pairs=(65, -1, 0, 0)), dict(scaling=4), dict(scaling=-1), dict(base=1.0),
    dict(base=float("nan")), dict(base=float("inf")), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")),
    dict(scaling=2, n_axes=2, pairs=(63, 1, 0, 0)), dict(scaling=3, original_tokens=0), dict(scaling=3, slow_turns=32.0),
    dict(scaling=3, slow_turns=-1.0), dict(magnitude=-1.0), dict(magnitude=float("inf")), dict(frequencies=[4.0] * 64),
    dict(frequencies=[float("nan")] * 64),
])
def test_refuses(lib, bad):
    assert _make(lib, **bad)[0] == 1                         # FK_ERR_CONFIG


def test_arguments_are_checked_before_any_pointer(lib):
    st, r = _make(lib)
    assert st == 0 and lib.fk_rotary_make(None, ctypes.byref(r)) == 2
    ref = ctypes.byref(r)
    good = [ref, 4, None, 0, 0, None, 128, 1, None, 128, None, 0, 0, None, 0, None]
    assert lib.fk_rotate(*good) == 2                         # null tensors
    for i, v, want in [(0, None, 2), (1, -1, 1), (1, 1 << 31, 1), (3, 2, 1), (4, 3, 1), (4, -1, 1), (7, 0, 1), (7, 1025, 1), (12, 3, 2), (12, -1, 1)]:
        a = list(good)
        a[i] = v
        assert lib.fk_rotate(*a) == want, (i, v)
    assert lib.fk_rotate(ref, 0, None, 0, 0, None, 0, 1, None, 0, None, 0, 0, None, 0, None) == 0
    assert lib.fk_rotary_tables(ref, 3, None, None, None, None) == 2 and lib.fk_rotary_tables(ref, 0, None, None, None, None) == 0
    r.dim = 100                                              # not what make makes
    assert lib.fk_rotate(*good) == 1 and lib.fk_rotary_tables(ref, 3, None, None, None, None) == 1


def test_binding_refuses():
    from paper_2605_09681_gb300 import FkError, Rotary
    for kw in [dict(axes=(64, 64)), dict(dim=48, axes=(32,)), dict(base=0.5), dict(scaling="linear", factor=0.0)]:
        with pytest.raises(FkError):
            Rotary(head_dim=128, **kw)
    for kw in [dict(axes=(16,) * 5), dict(frequencies=[1.0] * 63), dict(magnitude=0.0)]:
        with pytest.raises(ValueError):
            Rotary(head_dim=128, **kw)
    with pytest.raises(KeyError):
        Rotary(head_dim=128, layout="other")
