"""Linear attention with decays on the GPU against the recurrence in float64.

Bounds, per value, with |o| and |S| the sums of the terms' magnitudes (all from the oracle):
  S     what two fp32 roundings at every token come to (the oracle carries them along; chunks round less often), and 2^-18 |S|
        for decays (exp of a difference of sums, 2^-21), the three parts of a key and the sums over a chunk (64 of 2^-24).
  o     half a step of bf16 of the value (2^-8), and where tokens go through chunks the products q k and the states before them
        in bf16: half a step of each term, 2^-8 |o|; else what S's errors and D sums give: under 2^-14 |o|.
In the 2-norm of all outputs the chunks' two roundings and the last are independent: each is at most 2^-8 / sqrt(3) of its terms,
whose squares add up to those of o where signs are random, so together under 2^-8.
"""
import numpy as np
import pytest
import torch

from oracle import linear_state as R

pytestmark = pytest.mark.gpu


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).cuda()


def _dev(a):
    return torch.from_numpy(np.array(a, dtype=np.float32)).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _cache(**kw):
    from paper_2605_09681_gb300 import LinearStateCache
    base = dict(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=128, max_seqs=4)
    base.update(kw)
    return LinearStateCache(**base)


def _inputs(T, Hq, H, D, seed=0, decay="token", strong=0.0):
    r = np.random.default_rng(seed)
    q = R.to_bf16(r.standard_normal((T, Hq, D)).astype(np.float32))
    k = R.to_bf16((r.standard_normal((T, H, D)) * D ** -0.5).astype(np.float32))
    v = R.to_bf16((r.standard_normal((T, H, D)) * np.exp(0.5 * r.standard_normal((T, 1, 1)))).astype(np.float32))
    g = -np.logaddexp(0.0, r.standard_normal((T, H)) - 4.0 + 3.0 * strong).astype(np.float32)
    if decay == "head":
        g = np.broadcast_to(-np.exp2(-1.0 - 7.0 * r.random((1, H))).astype(np.float32), (T, H))
    return q, k, v, g, r.standard_normal((H, D, D)).astype(np.float32)


def _check(got_o, got_s, q, k, v, g, s0, scale=None, norm=True):
    """One sequence's outputs and state against the oracle's."""
    D = q.shape[2]
    o, s, oa, sa, e = R.attend(q, k, v, g, s0, D ** -0.5 if scale is None else scale)
    chunked = len(q) > 1
    assert (np.abs(got_s - s) <= 1.01 * e + 2.0 ** -18 * sa + 1e-30).all()
    bound = 2.0 ** -8 * np.abs(o) + ((2.0 ** -8 if chunked else 0.0) + 2.0 ** -14) * oa + 1e-30
    assert (np.abs(got_o - o) <= bound).all()
    if norm and o.size:
        assert np.linalg.norm(got_o - o) <= 2.0 ** -8 * np.linalg.norm(o)
        assert np.linalg.norm(got_s - s) <= 2.0 ** -20 * np.linalg.norm(s) + np.linalg.norm(e)


LENGTHS = [1, 2, 3, 5, 16, 17, 31, 33, 64, 100, 127, 128, 129, 191, 255, 256, 257, 385, 700]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", LENGTHS)
def test_one_sequence(T, D):
    q, k, v, g, s0 = _inputs(T, 2, 2, D, T)
    with _cache(head_dim=D) as cache:
        cache.states(0)[1] = _dev(s0)
        cache.step([1], [T])
        o = cache.attend(0, _bf16(q), _bf16(k), _bf16(v), _dev(g))
        assert cache.sync_status() == 0
        _check(_np(o), _np(cache.states(0)[1]), q, k, v, g, s0)
        assert (cache.states(0)[[0, 2, 3]] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (4, 1), (6, 2), (7, 7), (24, 8)])
def test_shared_heads(Hq, H, D):
    lens = [150, 1, 20]
    T = sum(lens)
    q, k, v, g, s0 = _inputs(T, Hq, H, D, Hq)
    with _cache(head_dim=D, n_q_heads=Hq, n_kv_heads=H) as cache:
        cache.states(0)[[2, 0, 3]] = _dev(np.stack([s0, 2 * s0, 0 * s0]))
        cache.step([2, 0, 3], lens)
        o = _np(cache.attend(0, _bf16(q), _bf16(k), _bf16(v), _dev(g), scale=0.7))
        assert cache.sync_status() == 0
        s, at = _np(cache.states(0)), 0
        for i, (seq, n) in enumerate(zip([2, 0, 3], lens)):
            p = slice(at, at + n)
            _check(o[p], s[seq], q[p], k[p], v[p], g[p], [s0, 2 * s0, 0 * s0][i], 0.7)
            at += n


@pytest.mark.parametrize("decay", ["head", "none", "strong", "growing"])
@pytest.mark.parametrize("T", [3, 300])
def test_decays(decay, T):
    q, k, v, g, s0 = _inputs(T, 2, 2, 128, 5, decay="head" if decay == "head" else "token", strong=2.0 if decay == "strong" else 0.0)
    if decay == "none":
        g = np.zeros_like(g)
    if decay == "growing":
        g = -0.1 * g
    if decay == "strong":                                    # memories of a token and less, and far below the fp32 range
        g = g * np.array([1.0, 40.0], dtype=np.float32)
    with _cache() as cache:
        cache.states(0)[0] = _dev(s0)
        cache.step([0], [T])
        o = cache.attend(0, _bf16(q), _bf16(k), _bf16(v), _dev(g[0]) if decay in ("head", "none") else _dev(g))
        assert cache.sync_status() == 0
        _check(_np(o), _np(cache.states(0)[0]), q, k, v, g, s0)


@pytest.mark.parametrize("T", [4, 300])
def test_states_that_start_anew(T):
    """g = -inf: nothing from before a token reaches it."""
    q, k, v, g, s0 = _inputs(T, 2, 2, 64, 6)
    g = g.copy()
    g[0, 0] = g[T // 2, 1] = g[T - 1, 0] = -np.inf
    if T > 200:
        g[100:140, 0] = -np.inf
    with _cache(head_dim=64) as cache:
        cache.states(0)[0] = _dev(s0)
        cache.step([0], [T])
        o = cache.attend(0, _bf16(q), _bf16(k), _bf16(v), _dev(g))
        _check(_np(o), _np(cache.states(0)[0]), q, k, v, g, s0)


def test_steps_go_on_from_one_another():
    """Lengths that take turns between the recurrence and chunks: as one sequence."""
    lens = [200, 1, 1, 17, 128, 3, 260, 1]
    T = sum(lens)
    q, k, v, g, _ = _inputs(T, 4, 2, 128, 9)
    with _cache(n_q_heads=4, n_layers=2) as cache:
        outs, at = [], 0
        for n in lens:
            cache.step([3], [n])
            p = slice(at, at + n)
            for layer in (0, 1):
                o = cache.attend(layer, _bf16(q[p]), _bf16(k[p]), _bf16(v[p]), _dev(g[p]))
            outs.append(_np(o))
            at += n
        _check(np.concatenate(outs), _np(cache.states(1)[3]), q, k, v, g, np.zeros((2, 128, 128)))
        assert torch.equal(cache.states(0), cache.states(1))
        cache.fork(0, 3)
        assert torch.equal(cache.states(0)[0], cache.states(0)[3]) and torch.equal(cache.states(1)[0], cache.states(1)[3])
        cache.drop(3)
        assert (cache.states(0)[3] == 0).all() and (cache.states(1)[3] == 0).all() and (cache.states(1)[0] != 0).any()


@pytest.mark.parametrize("lens", [[5, 0, 1], [300, 0, 2, 129]])
def test_states_that_stay(lens):
    T, n = sum(lens), len(lens)
    q, k, v, g, _ = _inputs(T, 2, 2, 128, 11)
    s0 = np.random.default_rng(3).standard_normal((n, 2, 128, 128)).astype(np.float32)
    order = list(range(n))[::-1]
    with _cache() as cache:
        cache.states(0)[order] = _dev(s0)
        before = cache.states(0).clone()
        cache.step(order, lens)
        args = (0, _bf16(q), _bf16(k), _bf16(v), _dev(g))
        out = torch.full((n, 2, 128, 128), np.nan, device="cuda")
        o1 = cache.attend(*args, state_out=out)
        assert torch.equal(cache.states(0), before)
        o2 = cache.attend(*args, advance=False)
        assert torch.equal(cache.states(0), before) and torch.equal(o1, o2)
        o3 = cache.attend(*args)
        assert torch.equal(o1, o3) and torch.equal(cache.states(0)[order], out)
        assert cache.sync_status() == 0
        at = 0
        for i, m in enumerate(lens):
            p = slice(at, at + m)
            _check(_np(o1)[p], _np(out[i]), q[p], k[p], v[p], g[p], s0[i])
            at += m


def test_slices_of_wide_rows_and_guard_values():
    """Q, K, V of one projection, O and decays in wider rows; values around the rows in use are left alone and unread."""
    T, Hq, H, D = 333, 4, 2, 64
    q, k, v, g, s0 = _inputs(T, Hq, H, D, 13)
    wide = torch.full((T + 256, (Hq + 2 * H) * D + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    part = wide[128: 128 + T]
    Q, K, V = (part[:, a * D: (a + n) * D].unflatten(1, (n, D)) for a, n in ((0, Hq), (Hq, H), (Hq + H, H)))
    Q.copy_(_bf16(q)), K.copy_(_bf16(k)), V.copy_(_bf16(v))
    G = torch.full((T, H + 3), float("nan"), device="cuda")
    G[:, 1: 1 + H] = _dev(g)
    O = torch.full((T + 4, Hq * D + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    with _cache(head_dim=D, n_q_heads=Hq) as cache:
        cache.states(0)[0] = _dev(s0)
        cache.step([0], [T])
        cache.attend(0, Q, K, V, G[:, 1: 1 + H], O=O[2: 2 + T, 8: 8 + Hq * D].unflatten(1, (Hq, D)))
        assert cache.sync_status() == 0
        _check(_np(O[2: 2 + T, 8: 8 + Hq * D].unflatten(1, (Hq, D))), _np(cache.states(0)[0]), q, k, v, g, s0)
    O[2: 2 + T, 8: 8 + Hq * D] = 7.0
    assert (O == 7.0).all()


@pytest.mark.parametrize("where,value", [(w, x) for w in "qkvg" for x in (np.inf, -np.inf, np.nan) if (w, x) != ("g", -np.inf)])
@pytest.mark.parametrize("T", [6, 290])
def test_infinities_and_nan_reach_no_token_before_them(T, value, where):
    """Tokens before one that is not finite, and other sequences, are as if it were another value; behind it the values that are
    finite in float64 are the oracle's."""
    lens, bad = [70, T, 40], 70 + T - 3 if T < 100 else 70 + 200
    n = sum(lens)
    q, k, v, g, _ = _inputs(n, 2, 2, 64, 15)
    g = g.copy()
    {"q": q, "k": k, "v": v, "g": g}[where][(bad, 1, 5) if where != "g" else (bad, 1)] = value
    with _cache(head_dim=64) as cache:
        cache.step([0, 1, 2], lens)
        o = _np(cache.attend(0, _bf16(q), _bf16(k), _bf16(v), _dev(g)))
        s, at = _np(cache.states(0)), 0
        assert cache.sync_status() == 0
    for i, m in enumerate(lens):
        p = slice(at, at + m)
        want, sw, oa, sa, e = R.attend(q[p], k[p], v[p], g[p], np.zeros((2, 64, 64)), 64 ** -0.5)
        fine = np.isfinite(oa)
        assert fine[: bad - at].all() and (i == 1 or fine.all())
        with np.errstate(invalid="ignore"):
            assert (np.abs(o[p] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * oa)[fine].all()
            assert not np.isfinite(o[p][~np.isfinite(want)]).any()
            if i != 1:
                assert (np.abs(s[i] - sw) <= 1.01 * e + 2.0 ** -18 * sa).all()
            else:
                assert not np.isfinite(s[i][~np.isfinite(sw)]).any()
        at += m


@pytest.mark.parametrize("T", [1, 7, 400])
def test_captured_steps_go_on_at_each_replay(T):
    q, k, v, g, _ = _inputs(T, 2, 2, 128, 17)
    args = (0, _bf16(q), _bf16(k), _bf16(v), _dev(g))
    with _cache() as cache, _cache() as plain:
        cache.step([2], [T])
        plain.step([2], [T])
        out = torch.empty(T, 2, 128, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attend(*args, O=out)
        assert (cache.states(0) == 0).all()
        for _ in range(3):
            graph.replay()
            want = plain.attend(*args)
            assert torch.equal(out, want) and torch.equal(cache.states(0), plain.states(0))


@pytest.mark.parametrize("T,segments", [(700, 1), (700, 2), (700, 3), (700, 6), (129, 2), (1500, 0), (3000, 5)])
@pytest.mark.parametrize("D,Hq,H", [(64, 2, 2), (128, 3, 1)])
def test_segments(T, segments, D, Hq, H):
    """However a sequence is split, beside others that are not, and whatever the state goes to."""
    lens = [130, T, 40]
    n = sum(lens)
    q, k, v, g, s0 = _inputs(n, Hq, H, D, T + segments)
    with _cache(head_dim=D, n_q_heads=Hq, n_kv_heads=H) as cache:
        cache.force_plan(16, segments)
        cache.states(0)[:3] = _dev(np.stack([s0, -s0, 3 * s0]))
        cache.step([2, 1, 0], lens)
        args = (0, _bf16(q), _bf16(k), _bf16(v), _dev(g))
        new = torch.empty(3, H, D, D, device="cuda")
        o1 = cache.attend(*args, state_out=new)
        o2 = cache.attend(*args)
        assert cache.sync_status() == 0
        assert torch.equal(o1, o2) and torch.equal(new, cache.states(0)[[2, 1, 0]])
        at = 0
        for i, m in enumerate(lens):
            p = slice(at, at + m)
            _check(_np(o1)[p], _np(new[i]), q[p], k[p], v[p], g[p], [3 * s0, -s0, s0][i])
            at += m


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("D", [64, 128])
def test_drafts_of_every_group_size(G, D):
    lens = [1, 2, 7, 8, 9, 17, 3]
    n = sum(lens)
    q, k, v, g, s0 = _inputs(n, 2 * G, 2, D, G)
    with _cache(head_dim=D, n_q_heads=2 * G, n_kv_heads=2, max_seqs=7) as cache:
        cache.force_plan(32)
        cache.states(0)[:] = _dev(s0)
        cache.step(list(range(7)), lens)
        o = _np(cache.attend(0, _bf16(q), _bf16(k), _bf16(v), _dev(g)))
        s, at = _np(cache.states(0)), 0
        for i, m in enumerate(lens):
            p = slice(at, at + m)
            want, sw, oa, sa, e = R.attend(q[p], k[p], v[p], g[p], s0, D ** -0.5)
            assert (np.abs(o[p] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -14 * oa).all()     # all in fp32
            assert (np.abs(s[i] - sw) <= 1.01 * e + 2.0 ** -22 * sa).all()
            at += m


def test_the_same_inputs_give_the_same_bits():
    lens = [900, 1, 33, 130]
    q, k, v, g, _ = _inputs(sum(lens), 4, 2, 128, 19)
    args = (0, _bf16(q), _bf16(k), _bf16(v), _dev(g))
    with _cache(n_q_heads=4) as cache:
        cache.step([0, 1, 2, 3], lens)
        o = cache.attend(*args, advance=False)
        for _ in range(5):
            assert torch.equal(cache.attend(*args, advance=False), o)


def test_other_streams():
    lens = [260, 3]
    q, k, v, g, _ = _inputs(sum(lens), 2, 2, 128, 21)
    args = (0, _bf16(q), _bf16(k), _bf16(v), _dev(g))
    with _cache() as cache:
        cache.step([0, 1], lens)
        want = cache.attend(*args, advance=False)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = cache.attend(*args, stream=s)
        assert cache.sync_status(stream=s) == 0
        assert torch.equal(got, want)


def test_more_sequences_than_a_launch_takes():
    n = 300
    lens = [1 + (i * 37) % 3 for i in range(n)]
    lens[5], lens[280] = 200, 150
    T = sum(lens)
    q, k, v, g, _ = _inputs(T, 1, 1, 64, 23)
    with _cache(n_q_heads=1, n_kv_heads=1, head_dim=64, max_seqs=n) as cache:
        order = list(np.random.default_rng(0).permutation(n))
        cache.step(order, lens)
        o = _np(cache.attend(0, _bf16(q), _bf16(k), _bf16(v), _dev(g)))
        s, at = _np(cache.states(0)), 0
        assert cache.sync_status() == 0
        for seq, m in zip(order, lens):
            p = slice(at, at + m)
            _check(o[p], s[seq], q[p], k[p], v[p], g[p], np.zeros((1, 64, 64)), norm=False)
            at += m


def test_refusals():
    from paper_2605_09681_gb300 import FkError
    T = 4
    q = torch.zeros(T, 4, 64, dtype=torch.bfloat16, device="cuda")
    k, g = q[:, :2].contiguous(), torch.zeros(T, 2, device="cuda")
    with _cache(n_q_heads=4, head_dim=64, n_layers=2) as cache:
        with pytest.raises(ValueError):
            cache.attend(0, q, k, k, g)                      # no step: no tokens
        cache.step([0, 1], [3, 1])
        assert cache.attend(1, q, k, k, g).shape == q.shape
        for seqs, n in [([0, 0], [1, 1]), ([4], [1]), ([-1], [1]), ([0], [-1]), ([0, 1, 2, 3, 0], [1] * 5), ([0], [1 << 29])]:
            with pytest.raises(FkError):
                cache.step(seqs, n)
        assert cache.attend(1, q, k, k, g).shape == q.shape  # the step before stands
        for args in [(q[:3], k, k, g), (q.float(), k, k, g), (q, q, k, g), (q, k, k.cpu(), g), (q, k, k, g.double()), (q, k, k, g[:3]),
                     (q, k, k, g[:, :1]), (q, k, k, g.cpu())]:
            with pytest.raises(ValueError):
                cache.attend(0, *args)
        with pytest.raises(ValueError):
            cache.attend(0, q, k, k, g, scale=0.0)
        new = torch.zeros(2, 2, 64, 64, device="cuda")
        for bad in (new[:1], new.bfloat16(), new.cpu(), new.transpose(2, 3)):
            with pytest.raises(ValueError):
                cache.attend(0, q, k, k, g, state_out=bad)
        for layer in (-1, 2):
            with pytest.raises(FkError):
                cache.attend(layer, q, k, k, g)
        with pytest.raises(FkError):                         # the cache's own memory
            cache.attend(0, q, k, k, g, state_out=cache.states(1)[:2])
        for o in (q, ):
            with pytest.raises(FkError):                     # O where Q is
                cache.attend(0, q, k, k, g, O=o)
        wide = torch.zeros(T, 6 * 64, dtype=torch.bfloat16, device="cuda")
        a, b = wide[:, :256].unflatten(1, (4, 64)), wide[:, 128:].unflatten(1, (4, 64))
        with pytest.raises(FkError):
            cache.attend(0, a, k, k, g, O=b)
        with pytest.raises(FkError):
            cache.attend(0, q, wide[:, 256:].unflatten(1, (2, 64)), k, g, O=b)
        assert cache.attend(0, q, wide[:, 256:].unflatten(1, (2, 64)), k, g, O=a).shape == q.shape
        for seq in (-1, 4):
            with pytest.raises(FkError):
                cache.drop(seq)
            with pytest.raises(FkError):
                cache.fork(0, seq)
        cache.step([], [])
        assert cache.attend(0, q[:0], k[:0], k[:0], g[:0]).shape == (0, 4, 64)
