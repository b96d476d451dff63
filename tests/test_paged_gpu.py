"""The paged 8-bit cache on the GPU against its CPU statement: held values and rotated queries bit for bit,
attention within a bound derived from its roundings.

Attention bound: O is rounded to bf16 (2^-9 |o|; 2^-8 with the rounding of a value that lies across a power of two), the
softmax numerators to f16 (2^-12 each, so 2^-12 max |v| at most), and the logits carry fp32 sums: 128 products of
magnitudes that add up to at most ~64 after scaling, 2^-24 each, in a tree of at most 128 terms, under 2^-11 max |v|
together.  So |error| <= 2^-8 |o| + 2^-10 max |v|.
"""
import numpy as np
import pytest
import torch

from oracle import paged_cache as P

pytestmark = pytest.mark.gpu


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).cuda()


def _np(t):
    return t.float().cpu().numpy()


def _cache(**kw):
    from paper_2605_09681_gb300 import PagedKVCache
    base = dict(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=128, page_tokens=64, n_pages=64, max_seqs=8,
                max_seq_tokens=2048, rope="half")
    base.update(kw)
    return PagedKVCache(**base)


def _tables(rows, dim, seed=5):
    a = np.random.default_rng(seed).uniform(-9, 9, (rows, dim // 2))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def _normal(r, shape, spread=1.0):
    """bf16 values whose size differs from token to token."""
    return P.to_bf16((r.standard_normal(shape) * np.exp2(spread * r.standard_normal((shape[0], 1, 1)))).astype(np.float32))


def _bound(o, v):
    return 2.0 ** -8 * np.abs(o) + 2.0 ** -10 * (np.abs(v).max() if v.size else 0.0)


# ---------------------------------------------------------------- append
APPEND = [  # page, D, Hq, Hkv, style, rotated channels, tokens of each step
    (64, 128, 4, 2, "half", 128, [1]),
    (64, 128, 4, 2, "half", 128, [63, 1, 1]),
    (64, 128, 4, 2, "interleaved", 128, [65, 200, 7]),
    (32, 64, 3, 3, "half", 32, [31, 2, 64, 1, 1]),
    (32, 64, 8, 1, "interleaved", 64, [5, 5, 5, 70]),
    (128, 128, 10, 2, "half", 48, [100, 28, 128, 1]),
    (128, 64, 2, 2, "interleaved", 16, [1] * 6 + [130]),
    (32, 128, 5, 1, "half", 64, [1000]),
    (128, 128, 1, 1, "half", 128, [257, 0, 127]),
]


@pytest.mark.parametrize("page,D,Hq,Hkv,style,R,steps", APPEND)
def test_held_values_and_rotated_queries_bit_for_bit(page, D, Hq, Hkv, style, R, steps):
    r = np.random.default_rng(11)
    n = sum(steps)
    K, V, Q = _normal(r, (n, Hkv, D)), _normal(r, (n, Hkv, D), 3.0), _normal(r, (n, Hq, D))
    K[n // 2:, 0] *= 0.0 if n > 100 else 1.0                 # blocks of zeros
    c, s = _tables(n, R)
    want_k = P.rotate(K, c, s, style)
    want_q = P.to_bf16(P.rotate(Q, c, s, style))
    cos, sin = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
    with _cache(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_tokens=page, rope=style) as cache:
        at = 0
        for b in steps:
            cache.step([3], [b])
            part = slice(at, at + b)
            qr = cache.append(0, _bf16(K[part]), _bf16(V[part]), cos, sin, Q=_bf16(Q[part]))
            at += b
            assert cache.length(3) == at
            assert np.array_equal(_np(qr), want_q[part])
            hk, hv = cache.read(0, whole=True)
            assert np.array_equal(_np(hk), P.held(want_k[:at], page))
            assert np.array_equal(_np(hv), P.held(V[:at], page))
            first = (at - b) // page * page
            hk, hv = cache.read(0)
            assert np.array_equal(_np(hk), P.held(want_k[:at], page)[first:])
            assert np.array_equal(_np(hv), P.held(V[:at], page)[first:])
        assert cache.sync_status() == 0


def test_repeated_append_replaces_the_step():
    r = np.random.default_rng(12)
    K, V = _normal(r, (150, 2, 128)), _normal(r, (150, 2, 128))
    with _cache() as cache:
        cache.step([0], [70])
        cache.append(0, _bf16(K[:70]), _bf16(V[:70]))
        for n in (5, 80):                                    # inside the open page, and over its end
            for big in (1e4, 1e-4, 1.0):                     # larger, smaller, then the real ones
                if big == 1e4:
                    cache.step([0], [n])
                cache.append(0, _bf16(K[70: 70 + n] * big), _bf16(V[70: 70 + n] * big))
            hk, hv = cache.read(0, whole=True)
            assert np.array_equal(_np(hk), P.held(K[:70 + n], 64)) and np.array_equal(_np(hv), P.held(V[:70 + n], 64))
            # go back to 70 tokens by starting again
            cache.drop(0)
            cache.step([0], [70])
            cache.append(0, _bf16(K[:70]), _bf16(V[:70]))
            cache.step([0], [0])
        hk, _ = cache.read(0, whole=True)
        assert np.array_equal(_np(hk), P.held(K[:70], 64))


def test_ragged_batch_positions_strides_and_two_layers():
    r = np.random.default_rng(13)
    lens = [[5, 64, 0, 33, 1], [1, 1, 40, 95, 0], [30, 0, 1, 1, 1]]
    Hq, Hkv, D = 6, 2, 64
    width = (Hq + 2 * Hkv) * D
    c, s = _tables(300, D)
    cos, sin = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
    held_k = [[np.zeros((0, Hkv, D), np.float32)] * 5 for _ in range(2)]
    held_v = [[np.zeros((0, Hkv, D), np.float32)] * 5 for _ in range(2)]
    seqs = [4, 0, 7, 2, 5]
    with _cache(n_layers=2, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_tokens=32) as cache:
        for n in lens:
            T = sum(n)
            cache.step(seqs, n)
            for layer in (1, 0):
                qkv = _normal(r, (T, Hq + 2 * Hkv, D))
                pos = r.integers(0, 300, T).astype(np.int32)
                x = _bf16(qkv).view(T, width)
                parts = [x[:, a * D: b * D].unflatten(1, (b - a, D)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv))]
                qr = cache.append(layer, parts[1], parts[2], cos, sin, torch.from_numpy(pos).cuda(), Q=parts[0], Q_out=parts[0])
                assert np.array_equal(_np(qr), P.to_bf16(P.rotate(qkv[:, :Hq], c[pos], s[pos], "half")))
                kr = P.rotate(qkv[:, Hq: Hq + Hkv], c[pos], s[pos], "half")
                at = 0
                for i, b in enumerate(n):
                    held_k[layer][i] = np.concatenate([held_k[layer][i], kr[at: at + b]])
                    held_v[layer][i] = np.concatenate([held_v[layer][i], qkv[at: at + b, Hq + Hkv:]])
                    at += b
                hk, hv = cache.read(layer, whole=True)
                assert np.array_equal(_np(hk), np.concatenate([P.held(x, 32) for x in held_k[layer]]))
                assert np.array_equal(_np(hv), np.concatenate([P.held(x, 32) for x in held_v[layer]]))
        assert cache.sync_status() == 0


def test_non_finite_values_and_positions_are_reported_and_contained():
    r = np.random.default_rng(14)
    K, V = _normal(r, (40, 2, 128)), _normal(r, (40, 2, 128))
    K[3, 0, 5], K[9, 1, 7], V[4, 0, 1], V[5, 1, 2] = np.inf, np.nan, -np.inf, np.nan
    with _cache() as cache:
        cache.step([0], [40])
        cache.append(0, _bf16(K), _bf16(V))
        hk, hv = cache.read(0)
        assert cache.sync_status() == 5 and cache.sync_status() == 0       # FK_ERR_RANGE, then cleared
        assert np.array_equal(_np(hk), P.held(K, 64)) and np.array_equal(_np(hv), P.held(V, 64))
        cache.step([1], [3])
        c, s = _tables(10, 128)
        pos = torch.tensor([2, 10, -1], dtype=torch.int32).cuda()
        cache.append(0, _bf16(K[10:13]), _bf16(V[10:13]), torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), pos)
        hk, _ = cache.read(0)
        assert cache.sync_status() == 5
        want = K[10:13].copy()
        want[:1] = P.rotate(want[:1], c[2:3], s[2:3], "half")
        assert np.array_equal(_np(hk), P.held(want, 64))


# ---------------------------------------------------------------- attention
def _attend(cache_kw, lens, n_query, masks, seed=21, spread=1.0, chunk=None, scale=None):
    """Fill sequences of `lens` tokens, ask n_query of each, compare under every mask."""
    r = np.random.default_rng(seed)
    kw = dict(n_q_heads=4, n_kv_heads=2, head_dim=128, page_tokens=64)
    kw.update(cache_kw)
    Hq, Hkv, D, page = kw["n_q_heads"], kw["n_kv_heads"], kw["head_dim"], kw["page_tokens"]
    T, N = sum(lens), sum(n_query)
    K, V, Q = _normal(r, (T, Hkv, D), 0.3), _normal(r, (T, Hkv, D), spread), _normal(r, (N, Hq, D), 0.5)
    pages = sum(-(-n // page) for n in lens) + 3
    with _cache(n_pages=pages, max_seqs=len(lens), max_seq_tokens=max(max(lens), 1), **kw) as cache:
        cache.step(range(len(lens)), lens, n_query)
        cache.append(0, _bf16(K), _bf16(V))
        at, qat, parts = 0, 0, []
        for n, m in zip(lens, n_query):
            parts.append((P.held(K[at: at + n], page), P.held(V[at: at + n], page), Q[qat: qat + m]))
            at, qat = at + n, qat + m
        q = _bf16(Q)
        for mask in masks:
            got = _np(cache.attend(0, q, scale=scale, **mask)).astype(np.float64)
            qat = 0
            for i, (k, v, x) in enumerate(parts):
                want = P.attention(x, k, v, mask.get("causal", True), mask.get("window", 0), mask.get("sinks", 0), scale)
                o = got[qat: qat + len(x)]
                bad = np.abs(o - want) > _bound(want, v)
                assert not bad.any(), (mask, i, int(bad.sum()), np.abs(o - want).max(), np.argwhere(bad)[:4].tolist())
                qat += len(x)
        assert cache.sync_status() == 0


ALL = [dict(), dict(causal=False), dict(window=50), dict(window=33, sinks=5), dict(window=1), dict(window=70, sinks=130),
       dict(causal=False, window=64, sinks=1)]

ATTEND = [  # heads, head_dim, page, lens, queries
    (4, 2, 128, 64, [1], [1]),
    (4, 2, 128, 64, [64, 65, 63], [1, 1, 1]),
    (8, 8, 128, 32, [300, 1, 0, 77], [1, 1, 1, 5]),
    (7, 1, 64, 32, [129, 500], [3, 9]),
    (16, 1, 128, 128, [200, 31], [1, 2]),
    (3, 3, 64, 128, [127, 128, 129], [17, 1, 40]),
    (40, 2, 64, 64, [260], [2]),
    (2, 2, 128, 64, [5, 10], [9, 20]),                     # queries before the first key
    (4, 2, 128, 32, [0, 0], [3, 1]),                       # nothing held
    (4, 2, 128, 64, [1500], [1]),                          # the key axis split
    (4, 1, 64, 32, [1900, 3, 700], [2, 1, 4]),
    (6, 3, 128, 64, [600, 90], [130, 90]),                 # chunks
    (5, 1, 128, 128, [400], [77]),
    (4, 4, 64, 64, [513, 40], [257, 33]),
]


@pytest.mark.parametrize("Hq,Hkv,D,page,lens,nq", ATTEND)
def test_attention_against_64_bits(Hq, Hkv, D, page, lens, nq):
    _attend(dict(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_tokens=page), lens, nq, ALL)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nq", [1, 40])
def test_value_blocks_of_very_different_size(D, nq):
    _attend(dict(head_dim=D, page_tokens=32), [330, 90], [nq, nq], [dict(), dict(causal=False)], spread=5.0)


def test_tiny_and_huge_magnitudes():
    r = np.random.default_rng(22)
    for nq in (1, 70):
        for kq, vv in ((1e-12, 1e-20), (1e12, 1e20), (1e-30, 1.0)):
            K, V, Q = (_normal(r, (n, h, 128), 0.2) for n, h in ((150, 2), (150, 2), (nq, 4)))
            K, V, Q = P.to_bf16(K * np.float32(1 / kq)), P.to_bf16(V * np.float32(vv)), P.to_bf16(Q * np.float32(kq))
            K[30:70], V[60:100] = 0, 0                     # blocks of zeros among them
            with _cache(page_tokens=32) as cache:
                cache.step([0], [150], [nq])
                cache.append(0, _bf16(K), _bf16(V))
                o = _np(cache.attend(0, _bf16(Q)))
            hk, hv = P.held(K, 32), P.held(V, 32)
            want = P.attention(Q, hk, hv, True, 0, 0)
            assert (np.abs(o - want) <= _bound(want, hv)).all(), (nq, kq, vv)


@pytest.mark.parametrize("scale", [0.02, 0.5])
def test_scale(scale):
    _attend({}, [200, 70], [3, 70], [dict(), dict(causal=False)], scale=scale)


def test_rows_of_masked_infinities_and_huge_keys():
    """What a query does not see never reaches it: infinities, NaN and large values at masked places."""
    r = np.random.default_rng(31)
    n, nq = 200, 150
    K, V, Q = _normal(r, (n, 2, 128), 0.3), _normal(r, (n, 2, 128)), _normal(r, (nq, 4, 128))
    K2, V2 = K.copy(), V.copy()
    K2[190:], V2[190:] = 3e38, 1e30
    K2[195, 0], V2[195, 1], V2[196, 0] = np.nan, np.inf, np.nan
    out = []
    for k, v in ((K, V), (K2, V2)):
        with _cache(page_tokens=32) as cache:
            cache.step([0], [n], [nq])
            cache.append(0, _bf16(k), _bf16(v))
            out.append(_np(cache.attend(0, _bf16(Q))))
    pos = n - nq + np.arange(nq)
    same = pos < 160                                       # their page's block is the same
    hk, hv = P.held(K, 32), P.held(V, 32)
    want = P.attention(Q, hk, hv, True, 0, 0)
    for o in out:
        assert (np.abs(o - want) <= _bound(want, hv))[same].all()
    hk2, hv2 = P.held(K2, 32), P.held(V2, 32)
    seen = pos < 190                                       # the block's other tokens, held more coarsely
    want2 = P.attention(Q, hk2, hv2, True, 0, 0)
    assert np.isfinite(out[1][seen]).all()
    assert (np.abs(out[1] - want2) <= _bound(want2, hv2[:190]))[seen].all()


def test_nan_query_stays_in_its_row():
    r = np.random.default_rng(32)
    for nq in (2, 60):
        K, V, Q = _normal(r, (90, 2, 128), 0.3), _normal(r, (90, 2, 128)), _normal(r, (nq, 4, 128))
        Q[1, 2, 7] = np.nan
        with _cache() as cache:
            cache.step([0], [90], [nq])
            cache.append(0, _bf16(K), _bf16(V))
            o = _np(cache.attend(0, _bf16(Q)))
        assert np.isnan(o[1, 2]).all()
        o[1, 2] = 0
        assert np.isfinite(o).all()


def test_slices_as_inputs_and_outputs():
    r = np.random.default_rng(33)
    K, V, Q = _normal(r, (100, 2, 128), 0.3), _normal(r, (100, 2, 128)), _normal(r, (100, 4, 128))
    with _cache() as cache:
        cache.step([0], [100])
        cache.append(0, _bf16(K), _bf16(V))
        plain = cache.attend(0, _bf16(Q))
        wide = torch.zeros((100, 10, 128), dtype=torch.bfloat16, device="cuda")
        wide[:, 1:5] = _bf16(Q)
        out = torch.full((100, 9, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        cache.attend(0, wide[:, 1:5], out[:, 3:7])
        assert torch.equal(out[:, 3:7], plain)
        assert (out[:, :3] == 7).all() and (out[:, 7:] == 7).all()


def test_results_do_not_change_from_run_to_run():
    r = np.random.default_rng(34)
    K, V, Q = _normal(r, (1900, 2, 128), 0.3), _normal(r, (1900, 2, 128)), _normal(r, (9, 4, 128))
    with _cache() as cache:
        cache.step([0], [1900], [9])
        cache.append(0, _bf16(K), _bf16(V))
        q = _bf16(Q)
        first = cache.attend(0, q)
        for _ in range(20):
            assert torch.equal(cache.attend(0, q), first)


# ---------------------------------------------------------------- steps
def test_decoding_token_by_token_equals_the_prompt_at_once():
    r = np.random.default_rng(41)
    n = 140
    K, V, Q = _normal(r, (n, 2, 128), 0.3), _normal(r, (n, 2, 128)), _normal(r, (n, 4, 128))
    with _cache() as cache:
        cache.step([1], [n])
        cache.append(0, _bf16(K), _bf16(V))
        held = cache.read(0, whole=True)
        for i in range(n):
            cache.step([0], [1])
            cache.append(0, _bf16(K[i: i + 1]), _bf16(V[i: i + 1]))
            o = _np(cache.attend(0, _bf16(Q[i: i + 1])))
            if i % 16 in (0, 15):
                hk, hv = P.held(K[: i + 1], 64), P.held(V[: i + 1], 64)
                want = P.attention(Q[i: i + 1], hk, hv, True, 0, 0)
                assert (np.abs(o - want) <= _bound(want, hv)).all()
        again = cache.read(0, whole=True)
        assert torch.equal(held[0], again[0]) and torch.equal(held[1], again[1])


def test_more_sequences_than_one_launch_takes():
    r = np.random.default_rng(42)
    B = 600
    lens = r.integers(0, 40, B)
    K, V, Q = _normal(r, (int(lens.sum()), 1, 64)), _normal(r, (int(lens.sum()), 1, 64)), _normal(r, (B, 2, 64))
    order = r.permutation(B)
    with _cache(n_q_heads=2, n_kv_heads=1, head_dim=64, page_tokens=32, n_pages=2 * B, max_seqs=B, max_seq_tokens=64) as cache:
        cache.step(order, lens, [1] * B)
        cache.append(0, _bf16(K), _bf16(V))
        o = _np(cache.attend(0, _bf16(Q)))
        hk, _ = cache.read(0, whole=True)
        at = 0
        for i, n in enumerate(lens):
            k, v = P.held(K[at: at + n], 32), P.held(V[at: at + n], 32)
            assert np.array_equal(_np(hk[at: at + n]), k)
            want = P.attention(Q[i: i + 1], k, v, True, 0, 0)
            assert (np.abs(o[i: i + 1] - want) <= _bound(want, v)).all(), i
            at += n


def test_pages_come_back_and_are_refused_when_taken():
    from paper_2605_09681_gb300 import FkError
    r = np.random.default_rng(43)
    x = _bf16(_normal(r, (200, 2, 128)))
    with _cache(n_pages=4, max_seqs=3, max_seq_tokens=200) as cache:
        cache.step([0], [200])
        assert cache.free_pages() == 0
        cache.step([0], [100])                              # nothing was appended: withdrawn
        assert cache.free_pages() == 2 and cache.length(0) == 100
        cache.append(0, x[:100], x[:100])
        with pytest.raises(FkError) as e:
            cache.step([1], [129])
        assert e.value.name == "FK_ERR_FULL" and cache.free_pages() == 2
        o = cache.attend(0, x[:100].repeat(1, 2, 1))        # the step before is still current
        assert torch.equal(cache.read(0)[0], cache.read(0, whole=True)[0]) and torch.isfinite(o).all()
        with pytest.raises(FkError) as e:
            cache.step([0], [101])                          # beyond max_seq_tokens
        assert e.value.name == "FK_ERR_FULL"
        cache.step([1], [128])
        cache.append(0, x[:128], x[:128])
        cache.drop(0)
        assert cache.free_pages() == 2 and cache.length(0) == 0 and cache.length(1) == 128
        cache.step([2], [65])
        cache.append(0, x[:65], x[:65])
        hk, _ = cache.read(0)
        assert np.array_equal(_np(hk), P.held(_np(x[:65]), 64))
        cache.step([1], [0])
        hk, _ = cache.read(0, whole=True)
        assert np.array_equal(_np(hk), P.held(_np(x[:128]), 64))


def test_refusals():
    from paper_2605_09681_gb300 import FkError
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    cos = torch.zeros((300, 64), device="cuda")

    def name(f):
        with pytest.raises(FkError) as e:
            f()
        return e.value.name

    with _cache(n_layers=2) as cache:
        assert name(lambda: cache.append(0, b(0, 2, 128), b(0, 2, 128))) == "FK_ERR_STATE"
        for seqs, new, nq in (([8], [1], None), ([-1], [1], None), ([1, 1], [1, 1], None), ([0], [-1], None), ([0], [1], [-1])):
            assert name(lambda: cache.step(seqs, new, nq)) == "FK_ERR_ARG"
        with pytest.raises(ValueError):
            cache.step([0, 1], [1])
        cache.step([0], [10])
        assert name(lambda: cache.attend(0, b(10, 4, 128))) == "FK_ERR_STATE"      # not appended to yet
        assert name(lambda: cache.read(0)) == "FK_ERR_STATE"
        assert name(lambda: cache.append(2, b(10, 2, 128), b(10, 2, 128))) == "FK_ERR_ARG"
        for K, V in ((b(9, 2, 128), b(10, 2, 128)), (b(10, 4, 128), b(10, 2, 128)), (b(10, 2, 64), b(10, 2, 64)),
                     (b(10, 2, 128).float(), b(10, 2, 128)), (b(10, 2, 128).cpu(), b(10, 2, 128)),
                     (b(10, 128, 2).transpose(1, 2), b(10, 2, 128))):
            with pytest.raises(ValueError):
                cache.append(0, K, V)
        kv = b(10, 2, 128)
        for args in (dict(cos=cos), dict(sin=cos), dict(cos=cos.double(), sin=cos.double()), dict(cos=cos, sin=cos[:9]),
                     dict(cos=cos, sin=cos, positions=torch.zeros(10, device="cuda")),
                     dict(cos=cos, sin=cos, positions=torch.zeros(9, device="cuda", dtype=torch.int32))):
            with pytest.raises(ValueError):
                cache.append(0, kv, kv, **args)
        assert name(lambda: cache.append(0, kv, kv, cos[:9].contiguous(), cos[:9].contiguous())) == "FK_ERR_ARG"  # too few rows
        odd = torch.zeros((300, 12), device="cuda")
        assert name(lambda: cache.append(0, kv, kv, odd, odd)) == "FK_ERR_CONFIG"  # 24 channels
        assert name(lambda: cache.append(0, kv, kv, Q=b(10, 4, 128))) == "FK_ERR_ARG"   # queries without a rotation
        assert name(lambda: cache.append(0, kv, kv, cos.cpu(), cos.cpu())) == "FK_ERR_ARG"
        shifted = torch.zeros(10 * 256 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(10, 2, 128)
        assert name(lambda: cache.append(0, shifted, kv)) == "FK_ERR_ARG"          # 8-byte aligned
        narrow = torch.zeros(10 * 260, dtype=torch.bfloat16, device="cuda").as_strided((10, 2, 128), (260, 128, 1))
        assert name(lambda: cache.append(0, narrow, kv)) == "FK_ERR_ARG"           # stride not a multiple of 8
        cache.append(0, kv, kv)
        assert name(lambda: cache.step([0], [1])) == "FK_ERR_STATE"                # layer 1 was left out
        assert name(lambda: cache.drop(0)) == "FK_ERR_STATE"
        cache.append(1, kv, kv)
        for args in (dict(window=-1), dict(sinks=-1), dict(scale=float("inf"))):
            assert name(lambda: cache.attend(0, b(10, 4, 128), **args)) == "FK_ERR_CONFIG"
        with pytest.raises(ValueError):
            cache.attend(0, b(10, 4, 128), scale=0.0)
        with pytest.raises(ValueError):
            cache.attend(0, b(9, 4, 128))
        assert name(lambda: cache.attend(-1, b(10, 4, 128))) == "FK_ERR_ARG"
        cache.step([0], [1])
        assert cache.length(0) == 11
    from paper_2605_09681_gb300 import PagedKVCache
    with pytest.raises(FkError):
        _cache(device=1 << 20)
    with pytest.raises(FkError):
        _cache(head_dim=96)


def test_another_stream_and_a_captured_graph():
    r = np.random.default_rng(44)
    K, V, Q = _normal(r, (300, 2, 128), 0.3), _normal(r, (300, 2, 128)), _normal(r, (7, 4, 128))
    k, v, q = _bf16(K), _bf16(V), _bf16(Q)
    torch.cuda.synchronize()
    hk, hv = P.held(K, 64), P.held(V, 64)
    want = P.attention(Q, hk, hv, True, 0, 0)
    side = torch.cuda.Stream()
    with _cache() as cache:
        with torch.cuda.stream(side):
            cache.step([0], [293])
            cache.append(0, k[:293], v[:293])
            cache.step([0], [7])
            cache.append(0, k[293:], v[293:])
            o = cache.attend(0, q)
        side.synchronize()
        assert (np.abs(_np(o) - want) <= _bound(want, hv)).all()
        # the step's calls as a graph: with other contents of the same tensors they give those
        kb, vb, qb = k[293:].clone(), v[293:].clone(), q.clone()
        ob = torch.empty_like(qb)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.append(0, kb, vb)
            cache.attend(0, qb, ob)
        K2, V2, Q2 = _normal(r, (7, 2, 128), 0.3), _normal(r, (7, 2, 128)), _normal(r, (7, 4, 128))
        kb.copy_(_bf16(K2)); vb.copy_(_bf16(V2)); qb.copy_(_bf16(Q2))
        for _ in range(3):
            g.replay()
        torch.cuda.synchronize()
        hk, hv = P.held(np.concatenate([K[:293], K2]), 64), P.held(np.concatenate([V[:293], V2]), 64)
        want = P.attention(Q2, hk, hv, True, 0, 0)
        assert (np.abs(_np(ob) - want) <= _bound(want, hv)).all()
        assert cache.sync_status() == 0
