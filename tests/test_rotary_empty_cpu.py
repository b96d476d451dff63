"""Rotations of no tokens: sizes and types are checked, pointers are not (an empty tensor has none).  No kernel runs."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2605_09681_gb300 import build, _lib
    build.build()
    return _lib.load()


@pytest.fixture(scope="module")
def rotation(lib):
    from paper_2605_09681_gb300._lib import FkRotary, FkRotaryConfig
    c = FkRotaryConfig(128, 128, 0, 1, (ctypes.c_int32 * 4)(64), 0, 0, 1e4, 1.0, 1.0, 32.0, 0.0, None)
    r = FkRotary()
    assert lib.fk_rotary_make(ctypes.byref(c), ctypes.byref(r)) == 0
    return r


@pytest.mark.parametrize("heads2", [0, 1, 8])
def test_no_tokens(lib, rotation, heads2):
    call = lambda x2, y2: lib.fk_rotate(ctypes.byref(rotation), 0, None, 0, 0, None, 512, 4, None, 512, x2, 128 * heads2, heads2,
                                        y2, 128 * heads2, None)
    assert call(None, None) == 0
    if heads2:
        assert call(256, None) == 0 and call(256, 512) == 0  # (an address that is not looked at)


def test_no_tokens_of_wrong_sizes(lib, rotation):
    for type_, heads, heads2 in [(3, 4, 2), (0, 0, 2), (0, 4, 1025), (0, 4, -1)]:
        assert lib.fk_rotate(ctypes.byref(rotation), 0, None, 0, type_, None, 512, heads, None, 512, None, 0, heads2, None, 0, None) == 1


def test_queries_without_keys_need_no_second_tensor(lib, rotation):
    """With tokens a tensor and its heads go together, as before."""
    for x2, heads2, y2 in [(None, 2, None), (256, 0, 256), (256, 2, None), (None, 0, 256)]:
        assert lib.fk_rotate(ctypes.byref(rotation), 3, None, 0, 0, None, 512, 4, None, 512, x2, 256, heads2, y2, 256, None) == 2
