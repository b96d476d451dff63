"""Running sums of decays that go far within a chunk: what tokens behind many resets see depends on their own short sums alone.

Each query meets one key and each value is 1, so that an output is one decay, rounded once to bf16 where it multiplies the
values and exact from there on: half a step of the value's binade, and 2^-14 of it for a sum of decays (two halves in fp16 of what fp32
leaves of sums up to 128 * 159 < 2^15: 2^-21 each), exp2 and the products (under 2^-20 together).
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("resets", [40, 63, 64, 70, 96, 100])
@pytest.mark.parametrize("D,reset,scale", [(64, -110.0, 1.0), (128, -np.inf, 1.0), (128, -300.0, 0.5), (64, -np.inf, 0.7)])
def test_slow_decays_behind_resets(D, resets, reset, scale):
    from paper_2605_09681_gb300 import LinearStateCache
    T, H = 128, 8
    g = np.full((T, H), reset, dtype=np.float32)
    g[resets:] = -0.02 * np.random.default_rng(resets).random((T - resets, H)).astype(np.float32)
    g[resets] = reset
    q = torch.zeros(T, 2 * H, D, device="cuda", dtype=torch.bfloat16)
    k = torch.zeros(T, H, D, device="cuda", dtype=torch.bfloat16)
    v = torch.ones_like(k)
    q[:, :, 0] = 1.0
    k[resets, :, 0] = 1.0                                    # the one key: of the last token that resets
    with LinearStateCache(n_layers=1, n_q_heads=2 * H, n_kv_heads=H, head_dim=D, max_seqs=1) as cache:
        cache.states(0).fill_(3.0)
        cache.step([0], [T])
        o = cache.attend(0, q, k, v, torch.from_numpy(g).cuda(), scale=scale).double().cpu().numpy()
        assert cache.sync_status() == 0
    g[resets] = 0.0
    want = float(np.float32(scale)) * np.exp(np.cumsum(g[resets:].astype(np.float64), 0))
    half = 2.0 ** (np.floor(np.log2(want)) - 8)
    assert (o[:resets] == 0).all()
    got = o[resets:].reshape(T - resets, H, 2, D)
    assert (got == got[:, :, :1, :1]).all()
    assert (np.abs(got[:, :, 0, 0] - want) <= half + 2.0 ** -14 * want).all()
