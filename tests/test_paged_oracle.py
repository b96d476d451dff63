"""The paged cache's oracle against independent statements: torch's E4M3 conversion, hand-worked blocks and masks."""
import numpy as np
import torch

from oracle import paged_cache as P


def test_e4m3_agrees_with_torch_conversion():
    x = np.random.default_rng(0).standard_normal(20000) * np.exp2(np.random.default_rng(1).integers(-12, 9, 20000))
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(P._e4m3(x.astype(np.float64)), want.astype(np.float64))


def test_block_exponent_by_hand():
    # 448 fits e = 0; 449 does not: e = 1, step 32 * 2; zeros alone stay zero
    x = np.zeros((3, 1, 2), np.float32)
    x[0, 0] = [448, 1]
    x[1, 0] = [449, 1]
    assert P.held(x[:1], 1)[0, 0].tolist() == [448, 1]
    assert P.held(x[1:2], 1)[0, 0].tolist() == [448, 1]
    assert P.held(x[:2], 2)[0, 0].tolist() == [448, 1]
    assert not P.held(x[2:], 1).any()
    y = np.array([[[np.inf, 3.0]], [[np.nan, -2.0]]], np.float32)
    h = P.held(y, 2)            # largest finite 3: e = -7, largest magnitude 3.5
    assert h[0, 0].tolist() == [3.5, 3.0] and h[1, 0].tolist() == [0.0, -2.0]


def test_bf16_rounding_agrees_with_torch():
    x = np.random.default_rng(2).standard_normal(10000).astype(np.float32)
    assert np.array_equal(P.to_bf16(x), torch.from_numpy(x).to(torch.bfloat16).float().numpy())


def test_rotation_keeps_pair_norms_and_styles_are_permutations():
    r = np.random.default_rng(3)
    x = r.standard_normal((5, 2, 64)).astype(np.float32)
    a = r.standard_normal((5, 16))
    c, s = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
    y = P.rotate(x, c, s, "half")
    assert np.allclose(y[..., :16] ** 2 + y[..., 16:32] ** 2, x[..., :16] ** 2 + x[..., 16:32] ** 2, atol=1e-5)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    perm = np.arange(32).reshape(2, 16).T.ravel()
    z = P.rotate(x[..., perm], c, s, "interleaved")
    assert np.array_equal(z, y[..., perm])


def test_masks_by_hand():
    k = np.zeros((6, 1, 2))
    v = np.arange(6.0)[:, None, None] * np.ones((1, 1, 2))
    q = np.zeros((2, 1, 2))
    f = lambda **kw: P.attention(q, k, v, **dict(dict(causal=True, window=0, sinks=0), **kw))[:, 0, 0].tolist()
    assert f() == [2.0, 2.5]                        # queries at 4 and 5
    assert f(causal=False) == [2.5, 2.5]
    assert f(window=2) == [3.5, 4.5]
    assert f(window=2, sinks=1) == [7 / 3, 3.0]
    q = np.zeros((8, 1, 2))                         # two queries before the first key
    assert f()[:3] == [0.0, 0.0, 0.0] and f()[7] == 2.5
