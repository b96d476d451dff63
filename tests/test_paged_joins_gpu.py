"""Joins of key splits in company: captured and replayed, between launches of another cache on the same stream, and in steps whose
single tokens and prompts are both split.  Values against 64 bits at the bound of test_paged_gpu, bits against calls by themselves."""
import numpy as np
import pytest
import torch

import test_paged_gpu as T
from test_paged_plans_gpu import _check, _filled

pytestmark = pytest.mark.gpu

# heads, head_dim, page, keys, queries: joined by the last CTA (8 rows), by a kernel for 16-row CTAs, for one query tile, for two
JOINED = [((8, 1), 128, 64, [20000], [1]), ((16, 1), 64, 32, [9000], [1]), ((24, 2), 64, 32, [2500, 700, 3300], [8, 1, 5]),
          ((8, 1), 128, 64, [6000], [40]), ((12, 12), 128, 128, [9000], [300])]


@pytest.mark.parametrize("heads,D,page,lens,nq", JOINED)
def test_a_captured_join(heads, D, page, lens, nq):
    cache, Q, held = _filled(np.random.default_rng(91), heads, D, page, lens, nq)
    r = np.random.default_rng(92)
    with cache:
        q, masks = T._bf16(Q), (dict(), dict(causal=False))
        outs = [torch.empty_like(q) for _ in masks]
        for m in masks:
            cache.attend(0, q, **m)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(2):
                for o, m in zip(outs, masks):
                    cache.attend(0, q, o, **m)
        for _ in range(3):
            Q2 = T._normal(r, Q.shape, 0.5)
            q.copy_(T._bf16(Q2))
            for _ in range(2):
                g.replay()
            torch.cuda.synchronize()
            for o, m in zip(outs, masks):
                assert torch.equal(o, cache.attend(0, q, **m))
                _check(T._np(o), Q2, held, lens, nq, m, None if sum(nq) < 50 else 9)
        assert cache.sync_status() == 0


def test_caches_that_take_turns_on_a_stream():
    """An early-launched join, then another cache's launches (and its joins), again and again: each waits for its own parts."""
    made = [_filled(np.random.default_rng(93 + i), *shape) for i, shape in enumerate(JOINED)]
    queries = [T._bf16(Q) for _, Q, _ in made]
    alone = []
    for (cache, _, _), q in zip(made, queries):
        alone.append(cache.attend(0, q))
        torch.cuda.synchronize()
    for order in (range(5), range(4, -1, -1), (1, 2, 1, 3, 0, 4, 3, 3, 2, 0)):
        outs = [(i, made[i][0].attend(0, queries[i])) for _ in range(6) for i in order]
        torch.cuda.synchronize()
        assert all(torch.equal(o, alone[i]) for i, o in outs)
    for cache, _, _ in made:
        assert cache.sync_status() == 0
        cache.close()


@pytest.mark.parametrize("heads,D,page", [((8, 1), 128, 64), ((16, 4), 64, 32)])
def test_a_step_of_single_tokens_and_prompts_that_are_both_split(heads, D, page):
    lens = [9000, 40, 7000, 1, 300, 6500]
    nq = [1, 40, 70, 1, 2, 1]
    cache, Q, held = _filled(np.random.default_rng(98), heads, D, page, lens, nq)
    with cache:
        q = T._bf16(Q)
        for mask in (dict(), dict(causal=False), dict(window=4000, sinks=5)):
            o = cache.attend(0, q, **mask)
            _check(T._np(o), Q, held, lens, nq, mask)
            for _ in range(5):
                assert torch.equal(cache.attend(0, q, **mask), o)
        assert cache.sync_status() == 0
