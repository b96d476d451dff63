"""Host-side checks of the paged cache's C ABI: validation, struct layouts, null arguments.  No kernel runs."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2605_09681_gb300 import build, _lib
    build.build()
    return _lib.load()


def _cfg(**kw):
    from paper_2605_09681_gb300._lib import FkPagedConfig
    base = dict(n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=128, page_tokens=64, n_pages=16, max_seqs=4,
                max_seq_tokens=512, rope_style=0, device=0)
    base.update(kw)
    return FkPagedConfig(**base)


def test_struct_layouts():
    from paper_2605_09681_gb300._lib import FkPagedConfig, FkRope
    assert ctypes.sizeof(FkPagedConfig) == 40
    assert ctypes.sizeof(FkRope) == 32 and FkRope.rows.offset == 24


def test_accepts(lib):
    for kw in [dict(), dict(head_dim=64, page_tokens=32), dict(page_tokens=128, rope_style=1), dict(n_q_heads=2),
               dict(n_kv_heads=1, n_q_heads=71), dict(n_layers=256, max_seqs=65536, max_seq_tokens=1 << 19),
               dict(n_pages=(1 << 24) - 1, n_kv_heads=2, page_tokens=64)]:
        c = _cfg(**kw)
        assert lib.fk_paged_validate_config(ctypes.byref(c)) == 0, kw


@pytest.mark.parametrize("bad", [
    dict(n_layers=0), dict(n_layers=257), dict(n_q_heads=7), dict(n_q_heads=1), dict(n_kv_heads=0),
    dict(n_kv_heads=129, n_q_heads=129), dict(n_q_heads=2048), dict(head_dim=96), dict(page_tokens=16),
    dict(page_tokens=256), dict(n_pages=0), dict(max_seqs=0), dict(max_seqs=65537), dict(max_seq_tokens=0),
    dict(rope_style=2), dict(rope_style=-1), dict(n_pages=1 << 24, n_kv_heads=2, page_tokens=64),
    dict(max_seqs=65536, max_seq_tokens=1 << 20),
])
def test_refuses(lib, bad):
    c = _cfg(**bad)
    assert lib.fk_paged_validate_config(ctypes.byref(c)) == 1      # FK_ERR_CONFIG


def test_null_arguments(lib):
    assert lib.fk_paged_validate_config(None) == 2
    c = _cfg()
    assert lib.fk_paged_create(ctypes.byref(c), None) == 2
    n = ctypes.c_int64(0)
    assert lib.fk_paged_step(None, 0, None, None, None, None) == 2
    assert lib.fk_paged_append(None, 0, None, 0, None, 0, None, None, 0, None, 0, None) == 2
    assert lib.fk_paged_attend(None, 0, None, 0, None, 0, 1, 0, 0, 0.0, None) == 2
    assert lib.fk_paged_read(None, 0, 0, None, None, 0, ctypes.byref(n), None) == 2
    assert lib.fk_paged_drop(None, 0) == 2 and lib.fk_paged_sync_status(None, None) == 2
    assert lib.fk_paged_length(None, 0) == -1 and lib.fk_paged_free_pages(None) == -1
    assert lib.fk_paged_reserved_bytes(None) == 0 and lib.fk_paged_launch_count(None) == 0
    lib.fk_paged_destroy(None)


@pytest.mark.skipif(os.path.exists("/dev/nvidia0"), reason="checks the no-GPU error path")
def test_create_without_gpu_fails_cleanly(lib):
    c, h = _cfg(), ctypes.c_void_p()
    assert lib.fk_paged_create(ctypes.byref(c), ctypes.byref(h)) == 7 and not h.value
