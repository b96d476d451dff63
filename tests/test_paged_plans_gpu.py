"""The paged attention under each of its plans: the key axis split and joined, one or two query tiles to a CTA, a
leftover wave split by itself, more key tiles than a CTA's ring of block numbers holds, blocks of very different size
handed over piece by piece.  Values are compared with 64 bits at the bound of test_paged_gpu (derived there); where a whole
result is too large for the oracle, at queries spread over it."""
import numpy as np
import pytest
import torch

import test_paged_gpu as T
from oracle import paged_cache as P

pytestmark = pytest.mark.gpu


def _filled(r, heads, D, page, lens, nq, spread=1.0):
    """A cache of one layer with the step appended: cache, Q, and each sequence's held keys and values."""
    Hq, Hkv = heads
    K, V = T._normal(r, (sum(lens), Hkv, D), 0.3), T._normal(r, (sum(lens), Hkv, D), spread)
    Q = T._normal(r, (sum(nq), Hq, D), 0.5)
    cache = T._cache(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_tokens=page, max_seqs=len(lens),
                     n_pages=sum(-(-n // page) for n in lens) + 1, max_seq_tokens=max(lens))
    cache.step(range(len(lens)), lens, nq)
    cache.append(0, T._bf16(K), T._bf16(V))
    at, held = 0, []
    for n in lens:
        held.append((P.held(K[at: at + n], page), P.held(V[at: at + n], page)))
        at += n
    return cache, Q, held


def _check(out, Q, held, lens, nq, mask, some=None):
    at = 0
    for (k, v), n, m in zip(held, lens, nq):
        pick = range(m) if some is None else sorted(set(np.linspace(0, m - 1, some).astype(int).tolist()))
        for i in pick if some is not None else [None]:
            if i is None:
                want, got = P.attention(Q[at: at + m], k, v, mask.get("causal", True), mask.get("window", 0), mask.get("sinks", 0)), out[at: at + m]
            else:                                          # query i alone: the keys up to its position are what it is asked over
                upto = n - m + i + 1 if mask.get("causal", True) else n
                if mask.get("causal", True):
                    want = P.attention(Q[at + i: at + i + 1], k[:upto], v[:upto], True, mask.get("window", 0), mask.get("sinks", 0))
                else:
                    want = P.attention(Q[at + i: at + i + 1], k, v, False, 0, 0)
                got = out[at + i: at + i + 1]
            assert (np.abs(got - want) <= T._bound(want, v)).all(), (mask, i, np.abs(got - want).max())
        at += m


FEW = [  # heads, head_dim, page, lens, queries: single tokens and drafts over long caches
    ((8, 1), 128, 64, [40000], [1]),
    ((12, 12), 64, 32, [30000], [1]),
    ((16, 2), 128, 128, [21001, 200, 9000], [1, 2, 2]),
    ((24, 2), 64, 32, [2500, 700, 3300, 1], [8, 1, 5, 1]),
]


@pytest.mark.parametrize("heads,D,page,lens,nq", FEW)
def test_few_rows_over_a_long_cache(heads, D, page, lens, nq):
    cache, Q, held = _filled(np.random.default_rng(71), heads, D, page, lens, nq)
    with cache:
        for mask in (dict(), dict(causal=False), dict(window=5000, sinks=70)):
            _check(T._np(cache.attend(0, T._bf16(Q), **mask)), Q, held, lens, nq, mask)
        assert cache.sync_status() == 0


CHUNKS = [
    ((8, 1), 128, 64, [6000], [40]),                       # one query tile's worth and more, keys split and joined
    ((8, 1), 128, 32, [3001], [13]),                       # 104 rows
    ((4, 2), 64, 128, [7000, 150], [70, 150]),
    ((12, 4), 128, 128, [2600, 131, 900], [300, 131, 1]),
]


@pytest.mark.parametrize("heads,D,page,lens,nq", CHUNKS)
def test_chunks_with_the_keys_split(heads, D, page, lens, nq):
    cache, Q, held = _filled(np.random.default_rng(72), heads, D, page, lens, nq)
    with cache:
        q = T._bf16(Q)
        for mask in (dict(), dict(causal=False), dict(window=1000), dict(window=64, sinks=300)):
            o = cache.attend(0, q, **mask)
            _check(T._np(o), Q, held, lens, nq, mask)
            assert torch.equal(o, cache.attend(0, q, **mask))
        assert cache.sync_status() == 0


@pytest.mark.parametrize("D", [64, 128])
def test_a_leftover_wave_is_split(D):
    """168 items of 256 rows: more than the 152 SMs take at once."""
    lens, nq = [700], [650]
    cache, Q, held = _filled(np.random.default_rng(73), (64, 8), D, 64, lens, nq)
    with cache:
        _check(T._np(cache.attend(0, T._bf16(Q), causal=False)), Q, held, lens, nq, dict(causal=False), 25)
        assert cache.sync_status() == 0


@pytest.mark.parametrize("page", [32, 128])
def test_more_key_tiles_than_the_ring_of_block_numbers(page):
    """8700 keys: 68 tiles of a CTA, with a row tile for each SM so that nothing is split."""
    lens, nq = [8700], [608]
    cache, Q, held = _filled(np.random.default_rng(74), (64, 8), 64, page, lens, nq, spread=2.0)
    with cache:
        for mask in (dict(causal=False), dict()):
            _check(T._np(cache.attend(0, T._bf16(Q), **mask)), Q, held, lens, nq, mask, 12)
        assert cache.sync_status() == 0


@pytest.mark.parametrize("D,page", [(128, 32), (64, 32), (128, 64), (64, 128)])
def test_chunks_over_blocks_of_very_different_size(D, page):
    lens, nq = [700, 260], [200, 260]
    cache, Q, held = _filled(np.random.default_rng(75), (4, 2), D, page, lens, nq, spread=6.0)
    with cache:
        for mask in (dict(), dict(causal=False), dict(window=90, sinks=40)):
            _check(T._np(cache.attend(0, T._bf16(Q), **mask)), Q, held, lens, nq, mask)
        assert cache.sync_status() == 0


@pytest.mark.parametrize("B", [1, 40])
@pytest.mark.parametrize("nq", [5, 9, 17, 32, 33])
def test_row_counts_between_the_kernels(B, nq):
    lens, q = [100 + 3 * i for i in range(B)], [nq] * B
    cache, Q, held = _filled(np.random.default_rng(76), (8, 2), 64, 32, lens, q)
    with cache:
        for mask in (dict(), dict(window=20, sinks=3)):
            _check(T._np(cache.attend(0, T._bf16(Q), **mask)), Q, held, lens, q, mask)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("nq", [1, 300])
def test_a_query_that_is_not_finite_stays_in_its_head(bad, nq):
    lens = [5000]                                          # split and joined
    cache, Q, held = _filled(np.random.default_rng(77), (4, 2), 128, 64, lens, [nq])
    at = nq // 2
    X = Q.copy()
    X[at, 1, 5] = bad
    with cache:
        o, plain = T._np(cache.attend(0, T._bf16(X))), T._np(cache.attend(0, T._bf16(Q)))
    assert np.isnan(o[at, 1]).all()
    o[at, 1] = plain[at, 1]
    assert np.isfinite(o).all()
    assert (np.abs(o - plain) <= 2 * T._bound(plain, held[0][1])).all()


def test_pages_beyond_four_gigabytes():
    """A page's codes whose offset does not fit 32 bits: 2 MB a page (128 heads of 128, 128 tokens), 2112 pages taken before."""
    H, D, page, fill = 128, 128, 128, 8192
    r = np.random.default_rng(78)
    some = T._normal(r, (64, H, D), 0.3)
    lens = [300, 40]
    K, V = T._normal(r, (300, H, D), 0.3), T._normal(r, (300, H, D))
    with T._cache(n_q_heads=H, n_kv_heads=H, head_dim=D, page_tokens=page, max_seqs=3, n_pages=2112 + 4,
                  max_seq_tokens=33 * fill) as cache:
        x = T._bf16(some).repeat(fill // 64, 1, 1)
        for _ in range(33):
            cache.step([0], [fill])
            cache.append(0, x, x)
        for seq, nq in ((1, 300), (2, 1)):
            n = lens[seq - 1]
            cache.step([seq], [n], [nq])
            cache.append(0, T._bf16(K[:n]), T._bf16(V[:n]))
            hk, hv = cache.read(0, whole=True)
            k, v = P.held(K[:n], page), P.held(V[:n], page)
            assert np.array_equal(T._np(hk), k) and np.array_equal(T._np(hv), v)
            Q = T._normal(r, (nq, H, D), 0.5)
            out = T._np(cache.attend(0, T._bf16(Q)))
            for h in (0, 57, 127):
                want = P.attention(Q[:, h: h + 1], k[:, h: h + 1], v[:, h: h + 1], True, 0, 0)
                assert (np.abs(out[:, h: h + 1] - want) <= T._bound(want, v)).all(), (seq, h)
        assert cache.free_pages() == 0 and cache.sync_status() == 0


@pytest.mark.parametrize("nq", [3, 200])
def test_the_widest_window_is_none(nq):
    """Queries before the first key: their position less the window would not fit 32 bits."""
    lens = [2]
    cache, Q, held = _filled(np.random.default_rng(79), (4, 2), 128, 64, lens, [nq])
    with cache:
        q = T._bf16(Q)
        plain = cache.attend(0, q)
        for window, sinks in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 30, 5)):
            assert torch.equal(cache.attend(0, q, window=window, sinks=sinks), plain), window
        _check(T._np(plain), Q, held, lens, [nq], dict())
        for bad in (dict(window=2 ** 31), dict(window=2 ** 32 + 5), dict(window=4, sinks=2 ** 31)):
            with pytest.raises(ValueError):
                cache.attend(0, q, **bad)


def test_outputs_made_for_slices_of_one_and_more_tokens():
    """Outputs that the binding makes are dense whatever the rows of Q lie in, also where a dimension is one."""
    r = np.random.default_rng(80)
    for Hq, Hkv, n in ((4, 2, 1), (1, 1, 7), (1, 1, 1), (4, 2, 9)):
        K, V, Q = T._normal(r, (n, Hkv, 64), 0.3), T._normal(r, (n, Hkv, 64)), T._normal(r, (n, Hq, 64))
        wide = torch.zeros((n, Hq + 3, 64), dtype=torch.bfloat16, device="cuda")
        wide[:, 2: 2 + Hq] = T._bf16(Q)
        c, s = (torch.from_numpy(t).cuda() for t in T._tables(16, 64))
        with T._cache(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=64) as cache:
            cache.step([0], [n])
            a = cache.append(0, T._bf16(K), T._bf16(V), c, s, Q=T._bf16(Q))
            b = cache.append(0, T._bf16(K), T._bf16(V), c, s, Q=wide[:, 2: 2 + Hq])
            assert torch.equal(a, b) and b.is_contiguous()
            assert torch.equal(cache.attend(0, a), cache.attend(0, torch.cat((a, a), 1)[:, Hq:]))
            hk, hv = cache.read(0)
            out = torch.empty_like(hk), torch.empty_like(hv)
            assert cache.read(0, K=out[0], V=out[1])[0] is out[0]
            assert torch.equal(hk, out[0]) and torch.equal(hv, out[1])
            with pytest.raises(ValueError):
                cache.read(0, K=torch.empty((n, Hkv + 1, 64), dtype=torch.bfloat16, device="cuda")[:, :Hkv] if n > 1 else hk.float())
