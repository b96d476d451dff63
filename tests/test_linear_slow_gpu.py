"""Slow decays over many chunks.

Without keys the state is its start times exp(T g).  A chunk's fp32 rounding of it differs from value to value (at most 2^-24, and
as often up as down), so that what all values have in common is the error of the factor.  Of exp(128 g) - 1: the product with log2 e,
its constant, the sum, ln 2 and its product (2^-24 each at most) and its series (2^-23), 2^-21.2 of T g together, which is at most 1.03; of
the factors as they are rounded: what one lacks is made up for by the next, so 2^-24 of their product, and as much for each of 8
segments where those are joined, 2^-21.  Together under 2^-20.  (Without that it would be up to 400 2^-25 = 2^-16.4.)
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
RATES = (-2.0e-5, -1.93e-5, -1.1e-6, 1.7e-5)


@pytest.mark.parametrize("segments", [1, 8])
@pytest.mark.parametrize("D", [64, 128])
def test_the_same_slow_decay_at_every_token(D, segments):
    from paper_2605_09681_gb300 import LinearStateCache
    T, H = 128 * 400, len(RATES)
    r = torch.Generator(device="cuda").manual_seed(D)
    q = torch.zeros(T, H, D, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(T, H, D, generator=r, device="cuda").bfloat16()
    g = np.array(RATES, dtype=np.float32)
    with LinearStateCache(n_layers=1, n_q_heads=H, n_kv_heads=H, head_dim=D, max_seqs=1) as cache:
        cache.force_plan(1, segments)
        s0 = torch.randn(H, D, D, generator=r, device="cuda")
        cache.states(0)[0] = s0
        cache.step([0], [T])
        cache.attend(0, q, q, v, torch.from_numpy(g).cuda())
        assert cache.sync_status() == 0
        s = cache.states(0)[0].double()
    want = s0.double() * torch.from_numpy(np.exp(T * g.astype(np.float64))).cuda()[:, None, None]
    off = ((s - want) / want).flatten(1)
    assert off.abs().max() <= 400 * 2.0 ** -24 + 2.0 ** -20
    assert off.mean(1).abs().max() <= 2.0 ** -20, off.mean(1)
