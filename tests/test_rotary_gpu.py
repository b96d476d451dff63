"""Rotary positions on the GPU against float64.

Bound: an angle of up to a quarter turn is off by three roundings to fp32 (1.5 pi 2^-24), sine and cosine by 2 steps (2^-22), each
product and the sum by 2^-24, so a rotated channel by (|a| + |b|) m (1.5 pi + 4 + 2) 2^-24 < (|a| + |b|) m 2^-20, and by half a
step of its type.  Frequencies in double precision: 2^-52 of an angle, 2^31 2^-52 at the farthest position (below
2^-20 too); both go into 2^-19.
"""
import numpy as np
import pytest
import torch

from oracle import linear_state as R

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _rotary(**kw):
    from paper_2605_09681_gb300 import Rotary
    return Rotary(**kw)


def _np(t):
    return t.double().cpu().numpy()


def _positions(r, T, axes, far):
    p = r.integers(0, far, (T, axes))
    return p, torch.from_numpy(p.astype(np.int32)).cuda()


def _check(y, x, angle, m, style, dtype):
    want = R.rotate(x, angle, m, style)
    size = R.rotate(np.abs(x), np.zeros_like(angle), 1.0, style)
    n = angle.shape[1]
    a, b = (slice(0, n), slice(n, 2 * n)) if style == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    both = np.zeros_like(size)
    both[..., a] = both[..., b] = size[..., a] + size[..., b]
    bound = 2.0 ** -19 * m * both + torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -24
    assert (np.abs(y - want) <= bound).all()
    assert np.array_equal(y[..., 2 * n:], x[..., 2 * n:])


CASES = [  # tokens, heads of Q and K, head_dim, rotated, pairs of each axis, type, farthest position
    (1, 1, 0, 128, 128, (64,), "bf16", 10),
    (3, 32, 8, 128, 128, (64,), "bf16", 1 << 17),
    (257, 12, 12, 128, 128, (22, 21, 21), "bf16", 2000),
    (1000, 5, 3, 64, 32, (16,), "f16", 1 << 31),
    (77, 2, 1, 64, 16, (8,), "f32", 1 << 31),
    (33, 3, 3, 96, 80, (13, 1, 26), "f32", 1 << 20),
    (5, 1, 7, 256, 256, (128,), "bf16", 1 << 24),
    (19, 4, 0, 40, 32, (4, 4, 4, 4), "f16", 300),
    (2049, 40, 8, 128, 64, (32,), "bf16", 1 << 20),
]


@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hk,D,dim,pairs,dtype,far", CASES)
def test_rotation(T, Hq, Hk, D, dim, pairs, dtype, far, style):
    r, t = np.random.default_rng(T), TYPES[dtype]
    rot = _rotary(head_dim=D, dim=dim, layout=style, axes=pairs)
    freq, m = R.frequencies(pairs)
    p, pos = _positions(r, T, len(pairs), far)
    angle = R.angles(p, pairs, freq)
    Q = torch.from_numpy(r.standard_normal((T, Hq, D)).astype(np.float32)).to(t).cuda()
    if not Hk:
        _check(_np(rot.rotate(pos, Q)), _np(Q), angle, m, style, t)
        return
    K = torch.from_numpy(r.standard_normal((T, Hk, D)).astype(np.float32)).to(t).cuda()
    q, k = rot.rotate(pos, Q, K)
    _check(_np(q), _np(Q), angle, m, style, t)
    _check(_np(k), _np(K), angle, m, style, t)
    # the other way, in place, out of one wide tensor
    wide = torch.cat([Q, K], 1)
    a, b = wide[:, :Hq], wide[:, Hq:]
    rot.rotate(pos, a, b, inverse=True, Q_out=a, K_out=b)
    _check(_np(a), _np(Q), -angle, m, style, t)
    _check(_np(b), _np(K), -angle, m, style, t)


@pytest.mark.parametrize("scaling,kw", [
    ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)), ("ramp", dict(factor=16.0, original_tokens=4096)),
    ("ramp", dict(factor=8.0, original_tokens=8192, slow_turns=1.0, fast_turns=4.0, magnitude=1.0))])
def test_scaled_tables(scaling, kw):
    r = np.random.default_rng(7)
    rot = _rotary(head_dim=128, base=500000.0, scaling=scaling, **kw)
    freq, m = R.frequencies((64,), 500000.0, scaling, kw["factor"], kw.get("original_tokens", 0), kw.get("slow_turns", 1.0),
                            kw.get("fast_turns", 32.0))
    m = kw.get("magnitude", m)
    p, pos = _positions(r, 513, 1, 1 << 22)
    angle = R.angles(p, (64,), freq)
    cos, sin = rot.tables(pos)
    assert cos.dtype == torch.float32 and cos.shape == (513, 64)
    assert np.abs(_np(cos) - m * np.cos(angle)).max() <= m * 2.0 ** -20
    assert np.abs(_np(sin) - m * np.sin(angle)).max() <= m * 2.0 ** -20


def test_negative_and_extreme_positions():
    rot = _rotary(head_dim=64)
    p = np.array([[-(2 ** 31)], [-1], [0], [1], [2 ** 31 - 1]])
    cos, sin = rot.tables(torch.from_numpy(p.astype(np.int32)).cuda())
    angle = R.angles(p, (32,), R.frequencies((32,))[0])
    assert np.abs(_np(cos) - np.cos(angle)).max() <= 2.0 ** -20 and np.abs(_np(sin) - np.sin(angle)).max() <= 2.0 ** -20
    assert (cos[2] == 1).all() and (sin[2] == 0).all()


def test_given_frequencies():
    freq = [(-1) ** i * 3.0 / (1 + i) for i in range(16)]
    rot = _rotary(head_dim=32, frequencies=freq, magnitude=0.5)
    p, pos = _positions(np.random.default_rng(2), 50, 1, 1000)
    cos, sin = rot.tables(pos[:, 0])
    angle = R.angles(p, (16,), freq)
    assert np.abs(_np(cos) - 0.5 * np.cos(angle)).max() <= 2.0 ** -21 and np.abs(_np(sin) - 0.5 * np.sin(angle)).max() <= 2.0 ** -21


def test_inverse_is_the_gradient():
    """Of sum(w * rotate(x)) with respect to x: by differences, whose rounding (x, y in fp32) is 2^-20 / step."""
    rot = _rotary(head_dim=64, dim=32, layout="interleaved")
    r = np.random.default_rng(3)
    p, pos = _positions(r, 6, 1, 5000)
    x = torch.from_numpy(r.integers(-4, 5, (6, 2, 64)).astype(np.float32)).cuda()
    w = torch.from_numpy(r.integers(-4, 5, (6, 2, 64)).astype(np.float32)).cuda()
    grad = rot.rotate(pos, w, inverse=True)
    for c in (0, 1, 17, 31, 32, 63):
        d = torch.zeros_like(x)
        d[:, :, c] = 1.0
        num = ((rot.rotate(pos, x + d) - rot.rotate(pos, x - d)) / 2 * w).sum(-1)
        assert (num - grad[:, :, c]).abs().max() <= 64 * 16 * 2.0 ** -19


def test_tables_feed_the_paged_cache():
    """PagedKVCache.append with the tables rotates as rotate does: both in fp32, the queries rounded once (half a step of bf16
    each, from values (|a| + |b|) 2^-19 apart)."""
    from paper_2605_09681_gb300 import PagedKVCache
    r = np.random.default_rng(4)
    rot = _rotary(head_dim=128, scaling="ramp", factor=4.0, original_tokens=2048)
    pos = torch.arange(40000, 40100, dtype=torch.int32, device="cuda")
    cos, sin = rot.tables(pos)
    Q, K, V = (torch.from_numpy(r.standard_normal((100, h, 128)).astype(np.float32)).to(torch.bfloat16).cuda() for h in (8, 2, 2))
    with PagedKVCache(n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=128, page_tokens=32, n_pages=8, max_seqs=1,
                      max_seq_tokens=200) as cache:
        cache.step([0], [100])
        rows = torch.arange(100, dtype=torch.int32, device="cuda")
        q = cache.append(0, K, V, cos, sin, rows, Q=Q)
        assert cache.sync_status() == 0
    want = _np(rot.rotate(pos, Q))
    size = np.abs(_np(Q))
    both = size + np.roll(size, 64, -1)
    assert (np.abs(_np(q) - want) <= 2.0 ** -7 * np.abs(want) + 2.0 ** -18 * both).all()


def test_streams_graphs_and_empty():
    rot = _rotary(head_dim=64)
    x = torch.randn(100, 3, 64, device="cuda").to(torch.bfloat16)
    pos = torch.arange(100, dtype=torch.int32, device="cuda")
    want = rot.rotate(pos, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = rot.rotate(pos, x, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rot.rotate(pos, x, Q_out=out)
    x.neg_()
    g.replay()
    assert torch.equal(out, -want)
    none = rot.rotate(pos[:0], x[:0])
    assert none.shape == (0, 3, 64) and rot.tables(pos[:0])[0].shape == (0, 32)


def test_refusals():
    from paper_2605_09681_gb300 import FkError
    rot = _rotary(head_dim=64)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (pos.long(), pos[:3], pos.cpu(), pos[:, None].expand(4, 2)):
        with pytest.raises(ValueError):
            rot.rotate(bad, x)
    for bad in (x.double(), x[:, :, :32], x[:3], x.cpu(), x.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            rot.rotate(pos, bad)
    with pytest.raises(ValueError):
        rot.rotate(pos, x, x.float())
    wide = torch.zeros(4, 2 * 64 + 4, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(FkError):                             # rows 8 bytes off a 16-byte boundary
        rot.rotate(pos, wide[:, :128].unflatten(1, (2, 64)))
    with pytest.raises(FkError):
        rot.rotate(pos, wide[:, 4:132].unflatten(1, (2, 64)))
