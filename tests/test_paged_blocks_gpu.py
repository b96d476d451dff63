"""The paged attention where the blocks of values differ in size, against 64 bits under a bound that goes by what each
query sees: a query whose keys lie in small blocks has to come out of them as well as one of large blocks, whatever else the
sequence holds.

Bound of o_d = sum_j w_j v_jd (w: softmax weights of the visible keys): bf16 rounds o to 2^-8 of it; numerators have f16's 11 bits,
2^-11 each; logits (query elements cut to 2^-17 of the largest in chunks, fp32 sums) move a weight by at most 2^-13, twice for
numerator and sum: together 2^-8 |o| + 2^-10 sum_j w_j |v_jd|.  Below f16's normal range a numerator is off by at most 2^-24 of the largest,
whose weight is max w, so 2^-24 max w sum_j |v_jd| on top; and what lies 2^-100 below the largest value seen may be lost.
"""
import numpy as np
import pytest
import torch

import test_paged_gpu as T
from oracle import paged_cache as P

pytestmark = pytest.mark.gpu


def exact(q, k, v, causal=True, window=0, sinks=0):
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
        top = np.array([np.abs(x[row]).max() if row.any() else 0.0 for row in see])
        o[:, h] = w @ x
        b[:, h] = 2.0 ** -8 * np.abs(o[:, h]) + 2.0 ** -10 * (w @ np.abs(x)) + 2.0 ** -100 * top[:, None]
        b[:, h] += 2.0 ** -24 * w.max(1, initial=0.0)[:, None] * (see @ np.abs(x))
    return o, b


def check(heads, D, page, V, nq, masks, seed=1, K=None, Q=None, repeat=1):
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
            want, bound = exact(Q, hk, hv, **mask)
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
