"""Linear attention and rotary positions as a generator uses them: many sequences of all lengths at once, hybrid layers over
two kinds of cache, drafts that are verified, captured steps, rows far apart, memory held.

A sequence's results depend on its own tokens, state and split alone, so beside others they are, bit for bit, what they are
by themselves; against float64 the bounds are those of test_linear_gpu.py.
"""
import numpy as np
import pytest
import torch

from oracle import linear_state as R

pytestmark = pytest.mark.gpu


def _cache(**kw):
    from paper_2605_09681_gb300 import LinearStateCache
    base = dict(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=128, max_seqs=4)
    base.update(kw)
    return LinearStateCache(**base)


def _tensors(T, Hq, H, D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    decay = -torch.nn.functional.softplus(n(T, H) - 4.0)
    return n(T, Hq, D).bfloat16(), (n(T, H, D) * D ** -0.5).bfloat16(), n(T, H, D).bfloat16(), decay


def _np(t):
    return t.double().cpu().numpy()


def _check(o, s, q, k, v, g, s0):
    """One sequence that went through chunks, against the oracle."""
    D = q.shape[2]
    want, sw, oa, sa, e = R.attend(_np(q), _np(k), _np(v), _np(g), _np(s0), D ** -0.5)
    assert (np.abs(_np(s) - sw) <= 1.01 * e + 2.0 ** -18 * sa + 1e-30).all()
    assert (np.abs(_np(o) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -14) * oa + 1e-30).all()


def _lengths(n, seed):
    """Ragged ones, some of a token and some long."""
    r = np.random.default_rng(seed)
    lens = [int(x) for x in r.integers(20, 420, n)]
    lens[1], lens[n // 2], lens[n - 2], lens[7] = 1, 1500, 900, 128
    return lens


@pytest.mark.parametrize("D,Hq,H", [(64, 8, 8), (128, 8, 8), (128, 16, 8), (64, 24, 8)])
@pytest.mark.parametrize("segments", [0, 1, 3])
def test_many_sequences_beside_one_another(D, Hq, H, segments):
    """More items than the GPU has SMs, so that CTAs take several, of different lengths, one after the other."""
    lens = _lengths(45, D + Hq)
    q, k, v, g = _tensors(sum(lens), Hq, H, D, D + Hq)
    with _cache(n_q_heads=Hq, n_kv_heads=H, head_dim=D, max_seqs=45) as cache, \
            _cache(n_q_heads=Hq, n_kv_heads=H, head_dim=D, max_seqs=45) as alone:
        cache.states(0).normal_(generator=torch.Generator(device="cuda").manual_seed(1))
        alone.states(0).copy_(cache.states(0))
        s0 = cache.states(0).clone()
        if segments:
            cache.force_plan(8, segments)
            alone.force_plan(8, segments)
        order = [int(x) for x in np.random.default_rng(5).permutation(45)]
        cache.step(order, lens)
        o = cache.attend(0, q, k, v, g)
        assert cache.sync_status() == 0
        at = 0
        for i, (seq, n) in enumerate(zip(order, lens)):
            p = slice(at, at + n)
            if segments == 1:                            # (else a step of its own may be split another way)
                alone.step([seq], [n])
                assert torch.equal(alone.attend(0, q[p], k[p], v[p], g[p]), o[p])
                assert torch.equal(alone.states(0)[seq], cache.states(0)[seq])
            if i % 5 == 4 or n > 450:
                h, G = i % H, Hq // H
                one, its = slice(h, h + 1), slice(h * G, (h + 1) * G)
                _check(o[p, its], cache.states(0)[seq, one], q[p, its], k[p, one], v[p, one], g[p, one], s0[seq, one])
            at += n
        assert alone.sync_status() == 0


@pytest.mark.parametrize("D,Hq,H,segments", [(64, 8, 8, 1), (128, 16, 8, 1), (128, 8, 8, 3)])
def test_values_not_finite_in_some_of_many(D, Hq, H, segments):
    """They reach no other sequence, head or earlier token, whichever CTAs go through them and how often."""
    lens = _lengths(45, D)
    q, k, v, g = _tensors(sum(lens), Hq, H, D, D)
    starts = np.concatenate(([0], np.cumsum(lens)))[:-1]
    w = v.clone()
    bad = {}                                             # sequence of the step -> first bad token, of head 2
    for i, x in zip(range(3, 45, 4), (np.inf, np.nan, -np.inf) * 4):
        bad[i] = (7 * i) % lens[i]
        w[int(starts[i]) + bad[i], 2, (5 * i) % D] = float(x)
    with _cache(n_q_heads=Hq, n_kv_heads=H, head_dim=D, max_seqs=45) as cache:
        cache.force_plan(8, segments)
        cache.step(list(range(45)), lens)
        fine = cache.attend(0, q, k, v, g, advance=False)
        new = torch.empty(45, H, D, D, device="cuda")
        o = cache.attend(0, q, k, w, g, state_out=new)
        cache.attend(0, q, k, v, g)
        assert cache.sync_status() == 0
        of_head = lambda x: x.unflatten(1, (H, Hq // H))[:, 2]
        others = [h for h in range(H) if h != 2]
        for i, (at, n) in enumerate(zip(starts, lens)):
            p = slice(int(at), int(at) + n)
            assert torch.equal(new[i, others], cache.states(0)[i, others])
            a, b = o[p].unflatten(1, (H, Hq // H)), fine[p].unflatten(1, (H, Hq // H))
            assert torch.equal(a[:, others], b[:, others])
            if i not in bad:
                assert torch.equal(o[p], fine[p]) and torch.equal(new[i], cache.states(0)[i])
                continue
            t = bad[i]
            x, y = of_head(o[p]), of_head(fine[p])
            c = t // 128 * 128
            assert torch.equal(x[:c], y[:c])
            assert torch.isfinite(x[:t].float()).all() and not torch.isfinite(x[t:, :, (5 * i) % D].float()).any()
            assert not torch.isfinite(new[i, 2, :, (5 * i) % D]).any()
            # other channels of v of that head: sums of finite terms
            keep = [d for d in range(D) if d != (5 * i) % D]
            assert torch.isfinite(x[..., keep].float()).all()
            if i % 3 == 0 and n < 450:
                heads = slice(2 * (Hq // H), 3 * (Hq // H))
                want, _, oa, _, _ = R.attend(_np(q[p][:, heads]), _np(k[p][:, 2:3]), np.nan_to_num(_np(w[p][:, 2:3]), posinf=0, neginf=0),
                                             _np(g[p][:, 2:3]), np.zeros((1, D, D)), D ** -0.5)
                # (where the chunk holds one, the part from before it is rounded once more: 2^-8 of its terms)
                lim = 2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 2.0 ** -13) * oa
                assert (np.abs(_np(x) - want) <= lim)[..., keep].all()


class _Hybrid:
    """Attention layers of a small generator, in turn linear and over the paged cache, projections left out: each layer's queries,
    keys and values are slices of rows that the layer before gave."""
    Hq, H, D, layers = 8, 4, 64, 4

    def __init__(self, seqs=4, tokens=512):
        from paper_2605_09681_gb300 import LinearStateCache, PagedKVCache, Rotary
        g = torch.Generator(device="cuda").manual_seed(3)
        w = self.Hq + 2 * self.H
        self.w = [(torch.randn(self.Hq * self.D, w * self.D, generator=g, device="cuda") * (self.Hq * self.D) ** -0.5).bfloat16()
                  for _ in range(self.layers)]
        self.rotary = Rotary(head_dim=self.D, dim=32, layout="interleaved", axes=(8, 8))
        self.linear = LinearStateCache(n_layers=2, n_q_heads=self.Hq, n_kv_heads=self.H, head_dim=self.D, max_seqs=seqs)
        self.paged = PagedKVCache(n_layers=2, n_q_heads=self.Hq, n_kv_heads=self.H, head_dim=self.D, page_tokens=64,
                                  n_pages=seqs * tokens // 64, max_seqs=seqs, max_seq_tokens=tokens)
        self.decay = -torch.exp2(-2.0 - torch.arange(self.H, device="cuda", dtype=torch.float32))

    def step(self, seqs, counts):
        self.linear.step(seqs, counts)
        self.paged.step(seqs, counts)

    def forward(self, x, positions, keep=None):
        """x [tokens, Hq D]; keep: the linear layers' inputs and outputs."""
        Hq, H = self.Hq, self.H
        for i, w in enumerate(self.w):
            qkv = (x @ w).view(len(x), Hq + 2 * H, self.D)
            q, k, v = qkv[:, :Hq], qkv[:, Hq: Hq + H], qkv[:, Hq + H:]
            if i % 2 == 0:
                self.rotary.rotate(positions, q, k, Q_out=q, K_out=k)
                o = self.linear.attend(i // 2, q, k, v, self.decay)
                if keep is not None:
                    keep.append((q, k, v, o))
            else:
                q1, k1 = self.rotary.rotate(positions, q, k)
                self.paged.append(i // 2, k1, v)
                o = self.paged.attend(i // 2, q1)
            x = torch.nn.functional.rms_norm(o.reshape(len(x), -1).float(), (Hq * self.D,)).bfloat16()
        return x

    def close(self):
        self.linear.close()
        self.paged.close()


def _at(counts, starts):
    p = torch.cat([torch.arange(s, s + n) for n, s in zip(counts, starts)]).int().cuda()
    return torch.stack((p // 10, p % 10), 1).contiguous()


def test_a_generator_of_hybrid_layers():
    """Prompts, single tokens, a fork and a dropped sequence; the linear layers against float64 over the whole text."""
    m = _Hybrid()
    g = torch.Generator(device="cuda").manual_seed(9)
    x = lambda n: torch.randn(n, m.Hq * m.D, generator=g, device="cuda").bfloat16()
    history, lens = {s: [] for s in range(4)}, [0] * 4

    def run(seqs, counts):
        m.step(seqs, counts)
        kept = []
        out = m.forward(x(sum(counts)), _at(counts, [lens[s] for s in seqs]), kept)
        assert torch.isfinite(out.float()).all()
        at = 0
        for s, n in zip(seqs, counts):
            history[s].append([tuple(y[at: at + n] for y in layer) for layer in kept])
            lens[s] += n
            at += n

    run([2, 0], [200, 37])
    run([0, 2], [1, 1])
    run([2, 3, 0], [1, 130, 9])
    m.linear.fork(1, 2)
    history[1], lens[1] = list(history[2]), lens[2]
    run([0, 1, 2, 3], [1, 1, 1, 1])
    m.linear.drop(0)
    m.paged.drop(0)
    history[0], lens[0] = [], 0
    run([0, 1, 2], [70, 5, 140])
    assert m.linear.sync_status() == 0 and m.paged.sync_status() == 0
    for s in range(4):
        for layer in range(2):
            q, k, v, o = (torch.cat([h[layer][j] for h in history[s]]) for j in range(4))
            d = m.decay.expand(len(q), m.H)
            _check(o, m.linear.states(layer)[s], q, k, v, d, torch.zeros(m.H, m.D, m.D))
    m.close()


def test_captured_hybrid_steps():
    """A decoding step of all layers in one graph: its replays are what the calls give by themselves."""
    a, b = _Hybrid(), _Hybrid()
    g = torch.Generator(device="cuda").manual_seed(2)
    prompt = torch.randn(150 + 33, a.Hq * a.D, generator=g, device="cuda").bfloat16()
    outs = []
    for m in (a, b):
        m.step([1, 3], [150, 33])
        outs.append(m.forward(prompt, _at([150, 33], [0, 0])))
    assert torch.equal(*outs)
    x, pos = outs[0][[149, 182]].clone(), _at([1, 1], [150, 33])
    want = []
    for m in (a, b):
        m.step([1, 3], [1, 1])
    want = b.forward(x, pos)                             # (also: the libraries' first use)
    torch.cuda.synchronize()
    states = a.linear.states(0).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = a.forward(x, pos)
    assert torch.equal(a.linear.states(0), states)       # captured, not run
    graph.replay()
    assert torch.equal(got, want)
    for layer in range(2):
        assert torch.equal(a.linear.states(layer), b.linear.states(layer))
    want = b.forward(x, pos)                             # the states go on; the paged cache's token is replaced
    graph.replay()
    assert torch.equal(got, want)
    a.close()
    b.close()


def test_drafts_verified():
    """Drafts are tried without a trace, or for the states behind them; as many tokens as were right are then taken in."""
    Hq, H, D = 4, 2, 128
    q, k, v, g = _tensors(16, Hq, H, D, 31)
    with _cache(n_q_heads=Hq, n_kv_heads=H, max_seqs=2) as cache, _cache(n_q_heads=Hq, n_kv_heads=H, max_seqs=2) as plain:
        cache.states(0).normal_(generator=torch.Generator(device="cuda").manual_seed(1))
        plain.states(0).copy_(cache.states(0))
        plain.force_plan(32)
        new = torch.empty(2, H, D, D, device="cuda")
        cache.step([1, 0], [8, 8])
        o = cache.attend(0, q, k, v, g, state_out=new)
        assert torch.equal(cache.states(0), plain.states(0))
        right = [3, 8]                                   # of sequence 1 three, of sequence 0 all
        rows = torch.cat((torch.arange(3), torch.arange(8, 16))).cuda()
        cache.states(0)[0].copy_(new[1])
        cache.step([1], [3])
        cache.attend(0, q[:3], k[:3], v[:3], g[:3])
        plain.step([1, 0], right)
        want = plain.attend(0, q[rows], k[rows], v[rows], g[rows])
        assert torch.equal(plain.states(0), cache.states(0)) and torch.equal(o[rows], want)
        assert cache.sync_status() == 0


@pytest.mark.parametrize("T", [1, 9, 260])
def test_rows_far_apart(T):
    """Tokens 2^24 elements apart: their offsets pass 32 bits."""
    apart, Hq, H, D = 1 << 24, 4, 2, 128
    q, k, v, g = _tensors(T, Hq, H, D, T)
    wide = torch.empty(T, apart, dtype=torch.bfloat16, device="cuda")
    at, parts = 0, []
    for n in (Hq, H, H, Hq):
        parts.append(wide[:, at: at + n * D].unflatten(1, (n, D)))
        at += n * D
    Q, K, V, O = parts
    Q.copy_(q), K.copy_(k), V.copy_(v)
    far = torch.empty(T, apart // 16, device="cuda")
    far[:, 5: 5 + H] = g
    from paper_2605_09681_gb300 import Rotary
    rotary = Rotary(head_dim=D)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    with _cache(n_q_heads=Hq, n_kv_heads=H) as cache, _cache(n_q_heads=Hq, n_kv_heads=H) as plain:
        for c in (cache, plain):
            c.step([2], [T])
        a, b = rotary.rotate(pos, q, k)
        rotary.rotate(pos, Q, K, Q_out=Q, K_out=K)
        assert torch.equal(Q, a) and torch.equal(K, b)
        want = plain.attend(0, a, b, v, g)
        cache.attend(0, Q, K, V, far[:, 5: 5 + H], O=O)
        assert torch.equal(O, want) and torch.equal(cache.states(0), plain.states(0))
        assert cache.sync_status() == 0


def test_nothing_is_allocated_after_creation():
    lens = [500, 3, 1, 130]
    q, k, v, g = _tensors(sum(lens), 4, 2, 64, 1)
    o, new = torch.empty_like(q), torch.empty(4, 2, 64, 64, device="cuda")
    cos, sin = (torch.empty(sum(lens), 32, device="cuda") for _ in range(2))
    from paper_2605_09681_gb300 import Rotary
    rotary = Rotary(head_dim=64)
    pos = torch.arange(sum(lens), dtype=torch.int32, device="cuda")
    with _cache(n_q_heads=4, head_dim=64, n_layers=2) as cache:
        held, used = cache.reserved_bytes(), None
        for i in range(4):
            rotary.rotate(pos, q, k, Q_out=q, K_out=k)
            rotary.tables(pos, cos=cos, sin=sin)
            cache.step([3, 1, 0, 2], lens)
            for layer in range(2):
                cache.attend(layer, q, k, v, g, O=o, state_out=new)
                cache.attend(layer, q, k, v, g, O=o)
            cache.fork(1, 2)
            cache.drop(2)
            assert cache.sync_status() == 0
            if i == 0:                                   # (the kernels are loaded at their first use)
                torch.cuda.synchronize()
                used = torch.cuda.mem_get_info()[0]
        assert torch.cuda.mem_get_info()[0] == used and cache.reserved_bytes() == held


def test_overlaps_are_refused():
    from paper_2605_09681_gb300 import FkError
    T, Hq, H, D = 8, 4, 2, 64
    q, k, v, g = _tensors(T, Hq, H, D, 1)
    with _cache(n_q_heads=Hq, head_dim=D, n_layers=2) as cache:
        cache.step([0, 1], [5, 3])
        flat = torch.zeros(1 << 16, device="cuda")
        new = flat[:2 * H * D * D].view(2, H, D, D)
        assert cache.attend(0, q, k, v, g, state_out=new).shape == q.shape
        inside = flat.view(torch.bfloat16)
        o = inside[64: 64 + T * Hq * D].view(T, Hq, D)
        kk = inside[64: 64 + T * H * D].view(T, H, D)
        for bad in (dict(O=o), dict(K=kk), dict(V=kk), dict(Q=o), dict(decay=flat[4: 4 + T * H].view(T, H)), dict(decay=flat[9: 9 + H])):
            with pytest.raises(FkError):
                cache.attend(0, **{**dict(Q=q, K=k, V=v, decay=g, state_out=new), **bad})
        for bad in (flat[40: 40 + T * H].view(T, H), flat[40: 40 + H]):
            with pytest.raises(FkError):
                cache.attend(0, q, k, v, bad, O=o)
        mine = cache.states(1).view(torch.bfloat16).flatten()[:T * Hq * D].view(T, Hq, D)
        with pytest.raises(FkError):
            cache.attend(0, q, k, v, g, O=mine)
        for plan in ((-1, 0), (0, -1)):
            with pytest.raises(FkError):
                cache.force_plan(*plan)
        assert cache.sync_status() == 0


@pytest.mark.parametrize("D,Hq,H", [(64, 6, 6), (128, 8, 4)])
def test_captured_steps_of_chunks_and_single_tokens(D, Hq, H):
    """Prompts, drafts and single tokens of one step run beside one another: replays, calls of several layers in a row and what
    follows them in the stream find all of it done."""
    lens = [1, 900, 3, 1, 200, 1, 0, 131] + [1] * 30
    q, k, v, g = _tensors(sum(lens), Hq, H, D, D)
    seqs = list(range(len(lens)))
    kw = dict(n_layers=3, n_q_heads=Hq, n_kv_heads=H, head_dim=D, max_seqs=len(lens))
    with _cache(**kw) as cache, _cache(**kw) as plain:
        for c in (cache, plain):
            c.step(seqs, lens)
        out = [torch.empty_like(q) for _ in range(3)]
        after = [torch.empty_like(q) for _ in range(3)]
        copies = [torch.empty_like(plain.states(0)) for _ in range(3)]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for layer in range(3):
                cache.attend(layer, q, k, v, g, O=out[layer])
                after[layer].copy_(out[layer])
                copies[layer].copy_(cache.states(layer))
        for _ in range(3):
            graph.replay()
            for layer in range(3):
                want = torch.empty_like(q)
                for i, at in zip(seqs, np.concatenate(([0], np.cumsum(lens)))):
                    if lens[i] > 0:                      # each by itself
                        p = slice(int(at), int(at) + lens[i])
                        plain.force_plan(8 if lens[i] < 8 else 1, 3 if lens[i] > 500 else 1)
                        plain.step([i], [lens[i]])
                        want[p] = plain.attend(layer, q[p], k[p], v[p], g[p])
                # (a prompt may be split another way: two results, each within 2^-8 and 2^-20 of the exact ones)
                assert (after[layer].float() - want.float()).norm() <= 2.0 ** -7 * want.float().norm()
                assert (copies[layer] - plain.states(layer)).norm() <= 2.0 ** -18 * plain.states(layer).norm()
                assert torch.equal(after[layer], out[layer])
        assert cache.sync_status() == 0 and plain.sync_status() == 0


def test_rotations_that_overlap_are_refused():
    from paper_2605_09681_gb300 import FkError, Rotary
    rotary = Rotary(head_dim=64)
    T = 8
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    wide = torch.randn(T, 6 * 64, device="cuda").bfloat16()
    q, k, v = (wide[:, a * 64: (a + 2) * 64].unflatten(1, (2, 64)) for a in (0, 2, 4))
    want = rotary.rotate(pos, q, k)
    got = rotary.rotate(pos, q, k, Q_out=v, K_out=k)         # other slices of the rows, or the input itself
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    near = wide[:, 64: 3 * 64].unflatten(1, (2, 64))
    flat = wide.flatten()
    ints = flat.view(torch.int32)[:T]
    dense = flat[: T * 128].view(T, 2, 64)
    for bad in (dict(Q_out=k), dict(Q_out=near), dict(K_out=q), dict(Q_out=v, K_out=v), dict(Q_out=dense), dict(Q_out=q, K_out=near)):
        with pytest.raises(FkError):
            rotary.rotate(pos, q, k, **bad)
    for bad in (dict(Q_out=q), dict(K_out=dense)):
        with pytest.raises(FkError):
            rotary.rotate(ints, q, k.clone(), **bad)
    cos, sin = (torch.empty(T, 32, device="cuda") for _ in range(2))
    with pytest.raises(FkError):
        rotary.tables(pos, cos=cos, sin=cos)
    with pytest.raises(FkError):
        rotary.tables(cos.view(torch.int32).flatten()[:T], cos=cos, sin=sin)


@pytest.mark.parametrize("D,G", [(64, 3), (128, 2)])
def test_values_not_finite_in_every_chunk(D, G):
    """NaN in one channel of all values from a token on, in a long run that is not split: the other channels as without."""
    T = 700
    q, k, v, g = _tensors(T, 2 * G, 2, D, G)
    with _cache(n_q_heads=2 * G, head_dim=D) as cache:
        cache.force_plan(8, 1)
        cache.step([0], [T])
        w = v.clone()
        w[5:, 1, 3] = float("nan")
        o, fine = cache.attend(0, q, k, w, g, advance=False), cache.attend(0, q, k, v, g, advance=False)
        assert cache.sync_status() == 0
        assert torch.equal(o[:, :G], fine[:, :G])
        assert o[5:, G:, 3].isnan().all() and o[:5, G:].isfinite().all()
        keep = [d for d in range(D) if d != 3]
        want, _, oa, _, _ = R.attend(_np(q[:, G:]), _np(k[:, 1:]), _np(v[:, 1:]), _np(g[:, 1:]), np.zeros((1, D, D)), D ** -0.5)
        lim = 2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 2.0 ** -13) * oa
        assert (np.abs(_np(o[:, G:]) - want) <= lim)[..., keep].all()
