"""Growth (g > 0) beside resets and beyond what exp(g) can be in fp32, by the recurrence and in chunks."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _run(q, k, v, g, s0):
    """One sequence: o, the state after it."""
    from paper_2605_09681_gb300 import LinearStateCache
    T, H, D = k.shape
    with LinearStateCache(n_layers=1, n_q_heads=q.shape[1], n_kv_heads=H, head_dim=D, max_seqs=1) as cache:
        cache.states(0)[0] = s0
        cache.step([0], [T])
        o = cache.attend(0, q, k, v, torch.from_numpy(g).cuda())
        assert cache.sync_status() == 0
        return o.double().cpu().numpy(), cache.states(0)[0].double().cpu().numpy()


def _inputs(T, D, seed):
    r = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=r, device="cuda")
    return n(T, 4, D).bfloat16(), (n(T, 2, D) * D ** -0.5).bfloat16(), n(T, 2, D).bfloat16(), n(2, D, D)


@pytest.mark.parametrize("grow", [np.inf, 200.0, 89.0])
@pytest.mark.parametrize("T,at,D", [(5, 1, 64), (5, 1, 128), (130, 3, 128), (300, 261, 64), (300, 100, 128)])
def test_what_grew_beyond_fp32_does_not_come_back(T, at, D, grow):
    """exp(g) of 88.73 and more is no fp32 number: nothing is finite from there on, however much decays behind it."""
    q, k, v, s0 = _inputs(T, D, T)
    g = np.full((T, 2), -60.0, dtype=np.float32)
    g[:at] = -0.01
    g[at, 1] = grow
    o, s = _run(q, k, v, g, s0)
    g[at, 1] = -60.0
    o1, s1 = _run(q, k, v, g, s0)
    assert np.isfinite(o[:at]).all() and np.isfinite(o[:, :2]).all() and np.isfinite(s[0]).all()
    assert (o[:, :2] == o1[:, :2]).all() and (s[0] == s1[0]).all()
    # (a chunk that grows takes its exponents from other differences: both are within 2^-8 of terms of about 1)
    assert np.linalg.norm(o[:at, 2:] - o1[:at, 2:]) <= 2.0 ** -7 * np.linalg.norm(o1[:at, 2:])
    assert not np.isfinite(o[at:, 2:]).any() and not np.isfinite(s[1]).any()


@pytest.mark.parametrize("each", [13.0, 20.0])
@pytest.mark.parametrize("T,at,D", [(12, 2, 64), (12, 2, 128), (200, 20, 64), (300, 250, 128)])
def test_nothing_from_before_a_reset_grows_back(T, at, D, each):
    """Behind g = -inf there are no keys, so that the state is zero, and stays it when it grows by exp(78).  By exp(120), which is no
    fp32 number, a chunk multiplies its zeros with infinity: they are 0 or NaN, and nothing else."""
    q, k, v, s0 = _inputs(T, D, T)
    k[at:] = 0.0
    g = np.full((T, 2), -0.01, dtype=np.float32)
    g[at] = -np.inf
    g[at + 1: at + 7] = each
    o, s = _run(q, k, v, g, s0)
    assert np.isfinite(o[:at]).all() and (o[:at] != 0).any()
    if each == 20.0 and T > 100:
        o, s = np.nan_to_num(o, nan=0.0), np.nan_to_num(s, nan=0.0)
    assert (o[at:] == 0).all() and (s == 0).all()


@pytest.mark.parametrize("each", [13.0, 20.0])
@pytest.mark.parametrize("T,at,D", [(12, 2, 64), (200, 20, 128), (300, 250, 64)])
def test_strong_decays_that_grow_back(T, at, D, each):
    """exp(-150) exp(65) = exp(-85) of the state, or nothing at all (exp(-150) is 0 in fp32); with exp(100), which is no fp32 number,
    also NaN in a chunk, whose keys are zeros."""
    q, k, v, s0 = _inputs(T, D, T)
    k.zero_()
    g = np.zeros((T, 2), dtype=np.float32)
    g[at], g[at + 1: at + 6] = -150.0, each
    o, s = _run(q, k, v, g, s0)
    if each == 20.0 and T > 100:
        o, s = np.nan_to_num(o, nan=0.0), np.nan_to_num(s, nan=0.0)
    assert (np.abs(s) <= np.exp(5 * each - 149.0) * np.abs(s0.double().cpu().numpy())).all()
    assert (np.abs(o[at + 5:]) <= 1e-18).all()
