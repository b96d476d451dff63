"""The paged attention where the blocks of values differ in size, against 64 bits under a bound that goes by what each
query sees: a query whose keys lie in small blocks has to come out of them as well as one of large blocks, whatever else the
sequence holds.

Bound of o_d = sum_j w_j v_jd (w: softmax weights of the visible keys): bf16 rounds o to 2^-8 of it; numerators have f16's 11 bits,
2^-11 each; logits (query elements cut to 2^-17 of the largest in chunks, fp32 sums) move a weight by at most 2^-13, twice for
numerator and sum: together 2^-8 |o| + 2^-10 sum_j w_j |v_jd|.  Below f16's normal range a numerator is off by at most 2^-24 of the largest,
whose weight is max w, so 2^-24 max w sum_j |v_jd| on top; what lies 2^-100 below the largest value of a page that the query sees
a key of (that key is held to 2^-19 of it) may be lost; and bf16's last step is 2^-133.
Blocks that are larger than others by more than their weights are smaller are kept by what they add, and their numerators then relative to
the block's own largest weight: 2^-21 of it (`own`) in place of that term.
"""
import numpy as np
import pytest
import torch

import test_paged_gpu as T
from oracle import paged_cache as P

pytestmark = pytest.mark.gpu


def exact(q, k, v, page, causal=True, window=0, sinks=0, own=False):
    """(o, bound) of q [n_q][Hq][D] over held k, v [n][Hkv][D], query i at n - n_q + i."""
    nq, Hq, D = q.shape
    n, Hkv = k.shape[:2]
    p, j = (n - nq + np.arange(nq))[:, None], np.arange(n)[None, :]
    see = np.broadcast_to(j <= p, (nq, n)) if causal else np.ones((nq, n), bool)
    if window > 0:
        see = see & ((j > p - window) | (j < sinks))
    o, b = np.zeros((nq, Hq, D)), np.zeros((nq, Hq, D))
    for h in range(Hq):
        x = v[:, h * Hkv // Hq].astype(np.float64)
        s = np.where(see, (q[:, h].astype(np.float64) @ k[:, h * Hkv // Hq].astype(np.float64).T) / np.sqrt(D), -np.inf)
        w = np.exp(s - np.max(s, axis=1, keepdims=True, initial=-1e300))
        t = w.sum(1, keepdims=True)
        w = w / np.where(t > 0, t, 1.0)
        top = np.zeros(nq)
        for i in range(0, n, page):
            top = np.maximum(top, see[:, i: i + page].any(1) * np.abs(x[i: i + page]).max())
        o[:, h] = w @ x
        b[:, h] = 2.0 ** -8 * np.abs(o[:, h]) + 2.0 ** -10 * (w @ np.abs(x)) + 2.0 ** -100 * top[:, None] + 2.0 ** -134
        if own:
            most = np.concatenate([np.broadcast_to(w[:, i: i + 32].max(1, keepdims=True), (nq, min(32, n - i))) for i in range(0, n, 32)], 1)
            b[:, h] += 2.0 ** -21 * (most * see) @ np.abs(x)
        else:
            b[:, h] += 2.0 ** -24 * w.max(1, initial=0.0)[:, None] * (see @ np.abs(x))
    return o, b


def check(heads, D, page, V, nq, masks, seed=1, K=None, Q=None, repeat=1, own=False):
    """V [n][Hkv][D] of one sequence, nq queries: every mask against `exact`, `repeat` calls alike."""
    Hq, Hkv = heads
    r = np.random.default_rng(seed)
    n = len(V)
    K = T._normal(r, (n, Hkv, D), 0.3) if K is None else K
    Q = T._normal(r, (nq, Hq, D), 1.0) if Q is None else Q
    V = P.to_bf16(V.astype(np.float32))
    hk, hv = P.held(K, page), P.held(V, page)
    with T._cache(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_tokens=page, max_seqs=1, n_pages=-(-n // page) + 1, max_seq_tokens=n) as cache:
        cache.step([0], [n], [nq])
        cache.append(0, T._bf16(K), T._bf16(V))
        q = T._bf16(Q)
        for mask in masks:
            out = cache.attend(0, q, **mask)
            for _ in range(repeat - 1):
                assert torch.equal(cache.attend(0, q, **mask), out), mask
            got = T._np(out).astype(np.float64)
            want, bound = exact(Q, hk, hv, page, own=own, **mask)
            bad = ~(np.abs(got - want) <= bound)
            at = np.argwhere(bad)[:1]
            assert not bad.any(), (mask, int(bad.sum()), at.tolist(), [(got[tuple(i)], want[tuple(i)], bound[tuple(i)]) for i in at])
        assert cache.sync_status() == 0


def by_block(r, n, H, D, block, sizes):
    """Normal values [n][H][D]; block b of `block` tokens is sizes[b % len(sizes)] times as large."""
    x = r.standard_normal((n, H, D))
    return x * np.array([sizes[j // block % len(sizes)] for j in range(n)])[:, None, None]


MASKS = [dict(), dict(causal=False), dict(window=90, sinks=40), dict(causal=False, window=300)]
A, B = 1.0, 2.0 ** 20
WITHIN = [  # page, sizes of blocks of 32 tokens: a tile of 128 keys has blocks alike and blocks far apart
    (64, [A, A, B, B]), (64, [B, B, A, A]), (64, [A, A, 0, 0, B, B]),
    (32, [A, A, A, B]), (32, [B, 0, 0, A]), (32, [0, A, A, B, B]), (32, [A, B, B, B, 0, 0, 0]),
]


@pytest.mark.parametrize("page,sizes", WITHIN)
@pytest.mark.parametrize("heads,D,n,nq", [((4, 2), 128, 900, 700), ((4, 1), 64, 1500, 300), ((8, 1), 128, 2600, 16)])
def test_parts_of_a_tile_that_share_a_reference(page, sizes, heads, D, n, nq):
    """Parts handed over one after the other without any warp having to rescale what it holds: the warps of a tile, which do
    different work under a mask, must not overtake one another.  Queries of very different size raise their maxima in different tiles."""
    r = np.random.default_rng(81)
    Q = T._normal(r, (nq, heads[0], D), 1.0) * np.where(np.arange(nq) // 32 % 2, 4.0, 0.25).astype(np.float32)[:, None, None]
    check(heads, D, page, by_block(r, n, heads[1], D, 32, sizes), nq, MASKS, Q=P.to_bf16(Q), repeat=8)


SHAPES = [  # heads, head_dim, page, keys, queries: 8 and 16 rows to a CTA, one and two query tiles; whole and split keys
    ((4, 2), 128, 32, 300, 3), ((8, 1), 64, 64, 4000, 1), ((16, 1), 128, 32, 3000, 1), ((24, 2), 64, 32, 900, 5),
    ((8, 1), 128, 64, 2600, 16), ((4, 2), 128, 32, 700, 300), ((4, 2), 64, 128, 1500, 260), ((8, 2), 64, 32, 4000, 150),
]
FAR = [[1e15, 1e-19], [100, 1e-34], [1, 1e-36, 1], [1e-34, 1e30], [1e-20, 1e20], [1e-12, 1e-24, 1e-36], [1e-30, 1e-15, 1, 1e15, 1e30]]


@pytest.mark.parametrize("heads,D,page,n,nq", SHAPES)
@pytest.mark.parametrize("sizes", FAR)
def test_blocks_far_apart(heads, D, page, n, nq, sizes):
    r = np.random.default_rng(82)
    masks = [dict(), dict(causal=False), dict(window=page), dict(window=n // 3, sinks=page // 2)]
    check(heads, D, page, by_block(r, n, heads[1], D, page, sizes), nq, masks)
    run = n // (2 * len(sizes)) + 1                        # as long runs, so that key splits and CTAs' parts differ as a whole
    check(heads, D, page, by_block(r, n, heads[1], D, run, sizes), nq, masks)


@pytest.mark.parametrize("heads,D,page,n,nq", SHAPES)
def test_blocks_of_any_size(heads, D, page, n, nq):
    for seed in range(4):
        r = np.random.default_rng(83 + seed)
        sizes = 10.0 ** r.uniform(-34, 34, 61) * (r.random(61) < 0.9)
        check(heads, D, page, by_block(r, n, heads[1], D, 32, sizes), nq, [dict(), dict(causal=False), dict(window=70, sinks=9)], seed)


@pytest.mark.parametrize("heads,D,page,n,nq", SHAPES)
@pytest.mark.parametrize("ratio", [2.0 ** 30, 2.0 ** 66, 2.0 ** 90])
def test_channels_that_large_blocks_leave_out(heads, D, page, n, nq, ratio):
    """Large blocks hold something in one channel only: the others' sums are the small blocks'."""
    r = np.random.default_rng(84)
    for sizes in ([1.0, ratio], [1 / ratio, 1.0], [ratio, 1.0, 1.0]):
        V = by_block(r, n, heads[1], D, page, sizes)
        V[np.array([sizes[j // page % len(sizes)] == max(sizes) for j in range(n)])[:, None] & np.ones((1, heads[1]), bool), 1:] = 0
        check(heads, D, page, V, nq, [dict(), dict(causal=False), dict(window=2 * page + 5)])


@pytest.mark.parametrize("heads,D,page,n,nq", SHAPES)
@pytest.mark.parametrize("bits", [20, 40, 60])
def test_large_blocks_of_small_weight(heads, D, page, n, nq, bits):
    """Blocks 2^bits larger whose weights are 2^bits smaller: both kinds make up the result."""
    r = np.random.default_rng(85)
    u = np.sign(r.standard_normal(D))
    large = np.array([j // page % 2 == 1 for j in range(n)])
    for first in (large, ~large):
        K = 0.02 * r.standard_normal((n, heads[1], D)) - first[:, None, None] * (bits * np.log(2) / np.sqrt(D)) * u
        Q = u * (1 + 0.1 * r.random((nq, heads[0], D)))
        Q *= np.sqrt(D) / (Q * u).sum(-1, keepdims=True) * np.sqrt(D)
        V = r.standard_normal((n, heads[1], D)) * np.where(first, 2.0 ** bits, 1.0)[:, None, None]
        check(heads, D, page, V, nq, [dict(), dict(causal=False), dict(window=3 * page)],
              K=P.to_bf16(K.astype(np.float32)), Q=P.to_bf16(Q.astype(np.float32)), own=True)


@pytest.mark.parametrize("heads,D,page,n,nq", SHAPES)
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_queries_that_are_not_finite_over_blocks_far_apart(heads, D, page, n, nq, bad):
    r = np.random.default_rng(86)
    V = P.to_bf16(by_block(r, n, heads[1], D, page, [1e-20, 1e20, 0, 1e-30]).astype(np.float32))
    K, Q = T._normal(r, (n, heads[1], D), 0.3), T._normal(r, (nq, heads[0], D), 1.0)
    at = (nq // 2, heads[0] - 1)
    X = Q.copy()
    X[at][3] = bad
    with T._cache(n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=D, page_tokens=page, max_seqs=1, n_pages=-(-n // page), max_seq_tokens=n) as cache:
        cache.step([0], [n], [nq])
        cache.append(0, T._bf16(K), T._bf16(V))
        for mask in (dict(), dict(window=page)):
            o = T._np(cache.attend(0, T._bf16(X), **mask))
            assert np.isnan(o[at]).all()
            want, bound = exact(Q, P.held(K, page), P.held(V, page), page, **mask)
            o[at], want[at] = 0, 0
            assert (np.abs(o - want) <= bound).all(), mask


@pytest.mark.parametrize("nq", [2, 9, 40, 300])
def test_steps_and_slices_over_blocks_far_apart(nq):
    """Several sequences (one of them empty, one with queries before its first key) of one step, into a slice of wider rows."""
    heads, D, page = (8, 2), 64, 32
    r = np.random.default_rng(87)
    lens, asks = [300, 0, 7, 90, 2000], [nq, 1, nq, 3, nq]
    K, Q = T._normal(r, (sum(lens), 2, D), 0.3), T._normal(r, (sum(asks), 8, D), 1.0)
    V = P.to_bf16(by_block(r, sum(lens), 2, D, 17, [1e-25, 1e10, 1.0, 0, 1e-3]).astype(np.float32))
    out = torch.full((sum(asks), 12, D), 7.0, dtype=torch.bfloat16, device="cuda")
    with T._cache(n_q_heads=8, n_kv_heads=2, head_dim=D, page_tokens=page, max_seqs=5, n_pages=90, max_seq_tokens=2000) as cache:
        cache.step([3, 0, 4, 1, 2], lens, asks)
        cache.append(0, T._bf16(K), T._bf16(V))
        for mask in (dict(), dict(causal=False), dict(window=33, sinks=2)):
            cache.attend(0, T._bf16(Q), out[:, 3:11], **mask)
            got, at, qat = T._np(out), 0, 0
            assert (got[:, :3] == 7).all() and (got[:, 11:] == 7).all()
            for n, m in zip(lens, asks):
                want, bound = exact(Q[qat: qat + m], P.held(K[at: at + n], page), P.held(V[at: at + n], page), page, **mask)
                assert (np.abs(got[qat: qat + m, 3:11] - want) <= bound).all(), (n, mask)
                at, qat = at + n, qat + m
        assert cache.sync_status() == 0


@pytest.mark.parametrize("heads,D,nq", [((4, 2), 128, 1), ((8, 1), 64, 2), ((8, 2), 128, 64), ((8, 2), 64, 70)])
@pytest.mark.parametrize("ratio", [2.0 ** 6, 2.0 ** 9, 2.0 ** 13])
def test_many_keys_of_small_weight_in_small_blocks(heads, D, nq, ratio):
    """One key of 16 holds nearly all the weight and a value of 0, the others share the rest, and the first value is larger than
    theirs: whatever page the numerators go by, those of 2^-20 have to count.  (As many sequences as fill the device, so that no keys are split.)"""
    n, B = 1500, 160
    r = np.random.default_rng(88)
    u = np.sign(r.standard_normal(D))
    K, V = np.zeros((n, heads[1], D)), 1.0 + 0.1 * r.random((n, heads[1], D))
    K[5::16] = 20 * np.log(2) / np.sqrt(D) * u
    V[5::16] = 0
    V[0] *= ratio
    K, V, Q = (P.to_bf16(np.ascontiguousarray(x, dtype=np.float32)) for x in (K, V, np.broadcast_to(u, (nq, heads[0], D))))
    with T._cache(n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=D, page_tokens=64, max_seqs=B, n_pages=24 * B, max_seq_tokens=n) as cache:
        cache.step(range(B), [n] * B, [nq] * B)
        cache.append(0, T._bf16(K).repeat(B, 1, 1), T._bf16(V).repeat(B, 1, 1))
        for mask in (dict(), dict(causal=False), dict(window=700, sinks=1)):
            got = T._np(cache.attend(0, T._bf16(Q).repeat(B, 1, 1), **mask))
            want, bound = exact(Q, P.held(K, 64), P.held(V, 64), 64, **mask)
            assert (np.abs(got[:nq] - want) <= bound).all() and np.array_equal(got[:nq], got[-nq:]), mask


@pytest.mark.parametrize("D,page,news", [(128, 64, [3, 5, 40]), (64, 32, [70, 1]), (128, 32, [1, 1, 1, 20, 8])])
def test_infinities_among_zeros(D, page, news):
    """A page whose finite values are all 0 holds an infinity as its largest magnitude, 448 2^-120, as any page does: what `read` gives is
    what the attention sees, however the tokens came, and until a token of ordinary size joins the page."""
    n = sum(news)
    K, V = np.zeros((n, 2, D), np.float32), np.zeros((n, 2, D), np.float32)
    K[0, 0, 3], K[1 % n, 1, 5], V[0, 0, 1], V[2 % n, 1, 7], V[2 % n, 1, 9] = np.inf, -np.inf, -np.inf, np.inf, np.nan
    K[n - 3, 0] = 1.5                                      # (in the last page)
    Q = P.to_bf16(np.random.default_rng(89).standard_normal((n, 4, D)).astype(np.float32))
    with T._cache(head_dim=D, page_tokens=page) as cache:
        at = 0
        for b in news:
            cache.step([0], [b])
            cache.append(0, T._bf16(K[at: at + b]), T._bf16(V[at: at + b]))
            at += b
            hk, hv = cache.read(0, whole=True)
            assert np.array_equal(T._np(hk), P.held(K[:at], page)) and np.array_equal(T._np(hv), P.held(V[:at], page))
            got = T._np(cache.attend(0, T._bf16(Q[at - b: at])))
            want, bound = exact(Q[at - b: at], P.held(K[:at], page), P.held(V[:at], page), page)
            assert (np.abs(got - want) <= bound).all()
        assert cache.sync_status() == 5


@pytest.mark.parametrize("Hq,Hkv,D,page,lens,nq", T.ATTEND)
@pytest.mark.parametrize("spread", [1.0, 5.0])
def test_every_query_by_what_it_sees(Hq, Hkv, D, page, lens, nq, spread):
    r = np.random.default_rng(90)
    K, V, Q = T._normal(r, (sum(lens), Hkv, D), 0.3), T._normal(r, (sum(lens), Hkv, D), spread), T._normal(r, (sum(nq), Hq, D), 0.5)
    with T._cache(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, page_tokens=page, n_pages=sum(-(-n // page) for n in lens) + 1,
                  max_seqs=len(lens), max_seq_tokens=max(max(lens), 1)) as cache:
        cache.step(range(len(lens)), lens, nq)
        cache.append(0, T._bf16(K), T._bf16(V))
        for mask in T.ALL:
            got, at, qat = T._np(cache.attend(0, T._bf16(Q), **mask)), 0, 0
            for n, m in zip(lens, nq):
                want, bound = exact(Q[qat: qat + m], P.held(K[at: at + n], page), P.held(V[at: at + n], page), page, **mask)
                assert (np.abs(got[qat: qat + m] - want) <= bound).all(), (mask, n)
                at, qat = at + n, qat + m
        assert cache.sync_status() == 0


@pytest.mark.parametrize("heads,D,page,n,nq", SHAPES)
@pytest.mark.parametrize("down,up,bits", [(30, 60, 0), (60, 40, 0), (60, 90, 0), (56, 90, 22), (90, 60, 10), (40, 85, 40)])
def test_what_has_been_lifted_outlasts_a_large_block(heads, D, page, n, nq, down, up, bits):
    """Ordinary pages, then tiny ones of most of the weight, for which O is lifted, then large ones that hold one channel only, at a weight of
    2^-bits: in the other channels the ordinary pages' sums remain, in one CTA's keys and across key splits."""
    r = np.random.default_rng(87)
    u = np.sign(r.standard_normal(D))
    Q = u * (1 + 0.1 * r.random((nq, heads[0], D)))
    Q *= np.sqrt(D) / (Q * u).sum(-1, keepdims=True) * np.sqrt(D)
    for block in (page, n // 6 + 1, n // 3 + 1):
        kind = np.arange(n) // block % 3
        K = 0.02 * r.standard_normal((n, heads[1], D)) - (np.array([5.0, 0.0, bits])[kind] * np.log(2) / np.sqrt(D))[:, None, None] * u
        V = r.standard_normal((n, heads[1], D)) * np.array([1.0, 2.0 ** -down, 2.0 ** up])[kind][:, None, None]
        V[kind == 2, :, 1:] = 0
        check(heads, D, page, V, nq, [dict(), dict(causal=False), dict(window=n // 2)],
              K=P.to_bf16(K.astype(np.float32)), Q=P.to_bf16(Q.astype(np.float32)))
