"""Host-side checks of the linear attention's C ABI: validation, struct layouts, null arguments.  No kernel runs."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2605_09681_gb300 import build, _lib
    build.build()
    return _lib.load()


def _cfg(**kw):
    from paper_2605_09681_gb300._lib import FkLinearConfig
    base = dict(n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=128, max_seqs=4, device=0)
    base.update(kw)
    return FkLinearConfig(**base)


def test_struct_layout():
    from paper_2605_09681_gb300._lib import FkLinearConfig
    assert ctypes.sizeof(FkLinearConfig) == 24


@pytest.mark.parametrize("good", [dict(), dict(head_dim=64), dict(n_q_heads=2), dict(n_q_heads=1024, n_kv_heads=1),
                                  dict(n_kv_heads=128, n_q_heads=128), dict(n_layers=256, max_seqs=65536)])
def test_accepts(lib, good):
    assert lib.fk_linear_validate_config(ctypes.byref(_cfg(**good))) == 0


@pytest.mark.parametrize("bad", [dict(n_layers=0), dict(n_layers=257), dict(n_q_heads=7), dict(n_q_heads=1), dict(n_kv_heads=0),
                                 dict(n_kv_heads=129, n_q_heads=129), dict(n_q_heads=2048), dict(head_dim=96),
                                 dict(head_dim=256), dict(max_seqs=0), dict(max_seqs=65537)])
def test_refuses(lib, bad):
    assert lib.fk_linear_validate_config(ctypes.byref(_cfg(**bad))) == 1      # FK_ERR_CONFIG


def test_null_arguments(lib):
    assert lib.fk_linear_validate_config(None) == 2
    c = _cfg()
    assert lib.fk_linear_create(ctypes.byref(c), None) == 2
    assert lib.fk_linear_step(None, 0, None, None) == 2
    assert lib.fk_linear_attend(None, 0, None, 0, None, 0, None, 0, None, 0, None, 0, 0.0, 0, None, None) == 2
    p = ctypes.c_void_p()
    assert lib.fk_linear_states(None, 0, ctypes.byref(p)) == 2
    assert lib.fk_linear_drop(None, 0, None) == 2 and lib.fk_linear_fork(None, 0, 0, None) == 2
    assert lib.fk_linear_sync_status(None, None) == 2
    assert lib.fk_linear_reserved_bytes(None) == 0 and lib.fk_linear_launch_count(None) == 0
    lib.fk_linear_destroy(None)


@pytest.mark.skipif(os.path.exists("/dev/nvidia0"), reason="checks the no-GPU error path")
def test_create_without_gpu_fails_cleanly(lib):
    c, h = _cfg(), ctypes.c_void_p()
    assert lib.fk_linear_create(ctypes.byref(c), ctypes.byref(h)) == 7 and not h.value


def test_oracle_against_the_sum_over_tokens():
    """The recurrence against its sums written out: o_t = scale (exp(G_t) q_t S_0 + sum_j exp(G_t - G_j) (q_t k_j) v_j).  Both in
    float64, of at most 30 terms: 2^-45 of the terms' magnitudes."""
    from oracle import linear_state as R
    r = np.random.default_rng(1)
    T, Hq, H, D = 9, 4, 2, 8
    q, k, v = (r.standard_normal((T, h, D)) for h in (Hq, H, H))
    g = -r.exponential(1.0, (T, H))
    s0 = r.standard_normal((H, D, D))
    o, s, oa, sa, _ = R.attend(q, k, v, g, s0, 0.3)
    G = np.cumsum(g, 0)
    for h in range(Hq):
        z = h // 2
        for t in range(T):
            want = np.exp(G[t, z]) * (q[t, h] @ s0[z])
            for j in range(t + 1):
                want = want + np.exp(G[t, z] - G[j, z]) * (q[t, h] @ k[j, z]) * v[j, z]
            assert (np.abs(o[t, h] - 0.3 * want) <= 2.0 ** -45 * oa[t, h]).all()
    for z in range(H):
        want = np.exp(G[-1, z]) * s0[z] + sum(np.exp(G[-1, z] - G[j, z]) * np.outer(k[j, z], v[j, z]) for j in range(T))
        assert (np.abs(s[z] - want) <= 2.0 ** -45 * sa[z]).all()
