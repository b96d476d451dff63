"""Rotary positions and linear attention with a decay for each head, as cases to be timed and compared.

A case is a plain dict.  `kind` says which operator one pass is:

  rotate    queries and keys [tokens][heads][dim] are rotated by their positions in one call: halves or interleaved
            pairs, a part of the head, several position axes, frequencies scaled for long contexts, either direction.
            Outputs: the rotated queries and keys.
  tables    cos and sin [tokens][pairs] in fp32 of the same angles.
  state     one layer's linear attention over a step's sequences: S_t = exp(g_t) S_(t-1) + k_t v_t^T,
            o_t = scale q_t S_t, every sequence going on from the state that it holds.  Outputs: o, and the states
            after the step.

Sequences are ragged: `news` is a text of whole numbers, the tokens of each sequence in the step; `held` says for each
whether it holds a state already (1) or starts (0).  The sizes are those of this repository's workloads (12 heads
of 128 channels, 1560 tokens a frame, chunks of 3 frames, 21 frames) and generic ones of language models;
`draw` spreads the same options over the whole range.
"""
import math

import torch

own = False

_ROTARY = {"q_heads": 12, "kv_heads": 12, "dim": 128, "rotary": 128, "layout": "half", "axes": "", "base": 10000.0,
           "scaling": "none", "factor": 1.0, "original": 0, "inverse": False, "type": "bf16", "first": 0}
_STATE = {"kind": "state", "q_heads": 12, "kv_heads": 12, "dim": 128, "decay": "token"}
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _text(values):
    return " ".join(str(int(v)) for v in values)


def _rotary(name, kind, tokens, **kw):
    return dict(_ROTARY, name=name, kind=kind, tokens=tokens, **kw)


def _state(name, news, held, **kw):
    return dict(_STATE, name=name, news=_text(news), held=_text(held), **kw)


def listed():
    return [
        # the smallest rotation: a few drafted tokens far into a stretched context (launch latency)
        _rotary("rotate_draft", "rotate", 4, q_heads=32, kv_heads=8, scaling="ramp", factor=8.0, original=8192, first=50000),
        # a 480P chunk of 3 frames as video models rotate it: interleaved pairs, each of frame, row and column
        # turning a part of them
        _rotary("rotate_chunk", "rotate", 4680, layout="interleaved", axes="22 21 21"),
        # a long prompt of grouped small heads, half of each head rotated, turned back (the direction of a gradient), fp16
        _rotary("rotate_prompt", "rotate", 40003, q_heads=32, kv_heads=8, dim=64, rotary=32, inverse=True, type="f16",
                scaling="base", factor=4.0),
        # tables of one step of a decoding batch, each stream at a place of its own
        _rotary("tables_step", "tables", 64, scaling="linear", factor=4.0, first=20000),
        # tables of a whole long context
        _rotary("tables_context", "tables", 131072),
        # the smallest step: one stream, one token
        _state("state_token", [1], [1]),
        # a decoding batch: 64 streams, one token each, every token with its own decay: 64 KB of state a head read and written
        _state("state_batch", [1] * 64, [1] * 64, q_heads=16, kv_heads=16),
        # a few drafted tokens per stream, small heads that share states
        _state("state_draft", [5, 1, 8, 3] * 4, [1] * 16, q_heads=32, kv_heads=8, dim=64),
        # a 480P chunk of 3 frames behind the frames before it, one decay a head
        _state("state_chunk", [4680], [1], decay="head"),
        # ragged prompts, grouped heads
        _state("state_prompts", [1777, 300, 2500, 4001, 512, 63, 129, 1000], [0, 0, 1, 0, 1, 0, 0, 0], q_heads=32, kv_heads=16),
        # a batch that decodes while new prompts come in, small heads
        _state("state_mixed", [1] * 20 + [777, 1, 1, 1500, 1, 2, 130] + [1] * 20, [1] * 20 + [0, 1, 1, 0, 1, 1, 0] + [1] * 20,
               q_heads=24, kv_heads=24, dim=64),
        # 21 frames of 480P in one stream (the largest): 12 heads do not fill the device by themselves
        _state("state_video", [32760], [0], decay="head"),
    ]


_MOST = 32760 * 12 * 128                             # channels of the largest case's queries


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "tables", "state", "state", "state"])
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    q = kv * rng.choice([1, 1, 2, 3, 4])
    if kind != "state":
        scaling = rng.choice(["none", "none", "linear", "base", "ramp"])
        c = dict(_ROTARY, kind=kind, q_heads=q, kv_heads=kv, dim=dim, rotary=dim // rng.choice([1, 1, 2, 4]),
                 layout=rng.choice(["half", "interleaved"]), base=rng.choice([10000.0, 500000.0]), scaling=scaling,
                 inverse=rng.random() < 0.3, type=rng.choice(["bf16", "bf16", "f16", "f32"]), first=log(1, 1 << 20))
        if scaling != "none":
            c["factor"], c["original"] = float(rng.choice([2, 4, 8, 32])), rng.choice([2048, 4096, 8192])
        if rng.random() < 0.3:
            p = c["rotary"] // 2
            a = p // 3
            c["axes"] = _text([p - 2 * a, a, a])
        c["tokens"] = log(1, 131072 if kind == "tables" else _MOST // ((q + kv) * dim))
        return c
    c = dict(_STATE, q_heads=q, kv_heads=kv, dim=dim, decay=rng.choice(["token", "token", "head"]))
    for _ in range(1000):
        style = rng.choice(["token", "few", "chunk", "chunk", "mixed"])
        seqs = log(1, 64)
        top = log(17, 20000)
        one = {"token": lambda: 1, "few": lambda: rng.randint(1, 16), "chunk": lambda: max(1, int(top * rng.uniform(0.2, 1.0))),
               "mixed": lambda: 1 if rng.random() < 0.7 else rng.randint(1, top)}[style]
        news = [one() for _ in range(seqs)]
        if seqs * max(news) * q * dim <= _MOST and seqs * kv * dim * dim <= 64 * 16 * 128 * 128:
            c["news"], c["held"] = _text(news), _text(rng.random() < 0.7 for _ in news)
            return c
    raise AssertionError("no case drawn")


# ---------------------------------------------------------------- inputs


def _ints(text):
    return [int(v) for v in text.split()]


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def _axes(c):
    return _ints(c["axes"]) or [c["rotary"] // 2]


def _raw_rotary(c, seed):
    """Queries, keys, and each token's position along each axis: places of a video (frame, row, column) where there are
    several axes, else of a text (a prompt's follow one another; a step's few tokens are anywhere)."""
    g, T = _generator(seed), c["tokens"]
    n = len(_axes(c))
    if n > 1:
        t = torch.arange(T, device="cuda") + (c["first"] % 1000 + int(seed) % 97) * 1560
        pos = torch.stack([t // 1560, t % 1560 // 52, t % 52][:n], 1)
    elif T <= 64:
        pos = c["first"] + torch.randint(0, 4096, (T, 1), generator=g, device="cuda")
    else:
        pos = c["first"] + int(seed) % 97 + torch.arange(T, device="cuda")[:, None]
    pos = pos.to(torch.int32)
    if c["kind"] == "tables":
        return None, None, pos
    t = _TYPES[c["type"]]
    return _normal((T, c["q_heads"], c["dim"]), g).to(t), _normal((T, c["kv_heads"], c["dim"]), g).to(t), pos


def _raw_state(c, seed):
    """Queries, keys of about unit length, values whose size differs from token to token, logarithms of the decays (one a
    head, from a few tokens' memory to hundreds; or of each token, most of them near 0), and the states held."""
    g = _generator(seed)
    news, held = _ints(c["news"]), _ints(c["held"])
    T, H, D = sum(news), c["kv_heads"], c["dim"]
    q = _normal((T, c["q_heads"], D), g).to(torch.bfloat16)
    k = (_normal((T, H, D), g) * D ** -0.5).to(torch.bfloat16)
    v = (_normal((T, H, D), g) * torch.exp(0.5 * _normal((T, 1, 1), g))).to(torch.bfloat16)
    slow = torch.arange(H, device="cuda", dtype=torch.float32) / max(1, H - 1)
    if c["decay"] == "head":
        decay = -torch.exp2(-1.0 - 8.0 * slow) * (0.9 + 0.2 * torch.rand((H,), generator=g, device="cuda"))
    else:
        decay = -torch.nn.functional.softplus(_normal((T, H), g) - 1.0 - 5.0 * slow)
    s = _normal((len(news), H, D, D), g) * torch.tensor(held, device="cuda", dtype=torch.float32)[:, None, None, None]
    return q, k, v, decay, s


def prepare(case, seed):
    c = case
    st = {"case": c}
    if c["kind"] != "state":
        st["q"], st["k"], st["pos"] = _raw_rotary(c, seed)
        if own:
            from paper_2605_09681_gb300 import Rotary

            st["rotary"] = Rotary(head_dim=c["dim"], dim=c["rotary"], layout=c["layout"], axes=_axes(c), base=c["base"],
                                  scaling=c["scaling"], factor=c["factor"], original_tokens=c["original"])
        else:
            st["freq"], st["magnitude"] = _frequencies(c)
        return st
    st["q"], st["k"], st["v"], st["decay"], s = _raw_state(c, seed)
    news = _ints(c["news"])
    if own:
        from paper_2605_09681_gb300 import LinearStateCache

        cache = LinearStateCache(n_layers=1, n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["dim"],
                                 max_seqs=len(news))
        cache.states(0).copy_(s)
        cache.step(list(range(len(news))), news)
        st["cache"], st["new"] = cache, s               # (the new states' memory, overwritten)
    else:
        st["states"] = s
        dev = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")  # noqa: E731
        st["batch"] = dev([i for i, n in enumerate(news) for _ in range(n)])
        st["place"] = dev([j for n in news for j in range(n)])
    return st


# ---------------------------------------------------------------- the plain form


def _frequencies(c):
    """Radians a position step of each pair in fp64, axis by axis, and what cos and sin are multiplied with."""
    out = []
    for p in _axes(c):
        d = 2 * p
        base = c["base"] * (c["factor"] ** (d / (d - 2)) if c["scaling"] == "base" else 1.0)
        f = base ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
        if c["scaling"] == "linear":
            f = f / c["factor"]
        if c["scaling"] == "ramp":                      # by the turns of a pair over the original context: 1 to 32
            keep = ((c["original"] * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
            f = f * keep + f / c["factor"] * (1.0 - keep)
        out.append(f)
    return torch.cat(out).cuda(), 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0


def _plain_tables(st):
    """cos and sin [tokens][pairs]; the angles in 64 bits."""
    c = st["case"]
    p = st["pos"].double().repeat_interleave(torch.tensor(_axes(c), device="cuda"), 1)
    angle = p * st["freq"]
    return (angle.cos() * st["magnitude"]).float(), (angle.sin() * st["magnitude"]).float()


def _plain_rotate(st):
    c, R = st["case"], st["case"]["rotary"]
    cos, sin = (x[:, None, :] for x in _plain_tables(st))
    sin = -sin if c["inverse"] else sin

    def turned(x):
        y = x.float()
        a, b = (y[..., : R // 2], y[..., R // 2: R]) if c["layout"] == "half" else (y[..., 0:R:2], y[..., 1:R:2])
        u, w = a * cos - b * sin, b * cos + a * sin
        z = torch.cat([u, w], -1) if c["layout"] == "half" else torch.stack([u, w], -1).flatten(-2)
        return torch.cat([z, y[..., R:]], -1).to(x.dtype)

    return turned(st["q"]), turned(st["k"])


def _plain_state(st):
    """Chunks of tokens: within one by a masked product of queries and keys, across them by the states that the chunks add,
    joined by one product with their decays."""
    c = st["case"]
    news = _ints(c["news"])
    B, most, H, G, D = len(news), max(news), c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    C = min(128, most)
    n = -(-most // C)
    at = (st["batch"], st["place"])

    def padded(x):                                      # [tokens][heads]... -> [B][heads][n][C]..., zeros behind a sequence
        y = torch.zeros((B, n * C) + x.shape[1:], dtype=x.dtype, device="cuda")
        y[at] = x
        return y.unflatten(1, (n, C)).movedim(3, 1)

    q, k, v = (padded(st[x].float()) for x in "qkv")
    q = q.unflatten(1, (H, G))
    g = st["decay"].double()
    g = padded(g if c["decay"] == "token" else g.expand(len(at[0]), H))      # [B][H][n][C]
    run = g.cumsum(3)                                   # up to and with a token, from its chunk's start
    i = torch.arange(C, device="cuda")
    later = i[:, None] < i[None, :]
    within = (run[..., :, None] - run[..., None, :]).masked_fill_(later, -math.inf).float().exp_()
    o = ((q @ k[:, :, None].transpose(-1, -2)) * within[:, :, None]) @ v[:, :, None]
    add = (k * (run[..., -1:] - run).float().exp_()[..., None]).transpose(-1, -2) @ v        # [B][H][n][D][D]
    ends = run[..., -1].cumsum(2)                       # [B][H][n]: up to and with a chunk
    r = torch.arange(n, device="cuda")
    after = r[:, None] < r[None, :]
    across = (ends[..., :, None] - ends[..., None, :]).masked_fill_(after, -math.inf).float().exp_()
    s0 = st["states"]
    s = (across @ add.flatten(3)).unflatten(3, (D, D)) + ends.float().exp_()[..., None, None] * s0[:, :, None]
    before = torch.cat([s0[:, :, None], s[:, :, :-1]], 2)
    o += (q * run.float().exp_()[:, :, None, ..., None]) @ before[:, :, None]
    o = o.flatten(1, 2).movedim(1, 3).flatten(1, 2)[at] * D ** -0.5
    return o.to(torch.bfloat16), s[:, :, -1]


def run(state):
    c = state["case"]
    if not own:
        return {"rotate": _plain_rotate, "tables": _plain_tables, "state": _plain_state}[c["kind"]](state)
    if c["kind"] == "rotate":
        return state["rotary"].rotate(state["pos"], state["q"], state["k"], inverse=c["inverse"])
    if c["kind"] == "tables":
        return state["rotary"].tables(state["pos"])
    o = state["cache"].attend(0, state["q"], state["k"], state["v"], state["decay"], state_out=state["new"])
    return o, state["new"]


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    c = case
    D = c["dim"]
    if c["kind"] == "tables":
        pairs = c["rotary"] // 2
        return {"bytes": c["tokens"] * (4 * len(_axes(c)) + 8 * pairs), "flops": c["tokens"] * pairs * 3}
    heads = c["q_heads"] + c["kv_heads"]
    if c["kind"] == "rotate":
        row = heads * D * torch.finfo(_TYPES[c["type"]]).bits // 8
        return {"bytes": c["tokens"] * (2 * row + 4 * len(_axes(c))), "flops": c["tokens"] * heads * c["rotary"] * 3}
    news, held = _ints(c["news"]), _ints(c["held"])
    T = sum(news)
    decays = 4 * c["kv_heads"] * (T if c["decay"] == "token" else 1)
    states = 4 * c["kv_heads"] * D * D * (sum(held) + len(held))
    # a token of one head by the recurrence: its state decayed, the outer product added; its queries' products
    return {"bytes": T * 4 * heads * D + decays + states, "flops": T * D * D * (3 * c["kv_heads"] + 2 * c["q_heads"])}


# ---------------------------------------------------------------- the definition in 64 bits


def _exact_rotary(c, seed):
    q, k, pos = _raw_rotary(c, seed)
    at, turns = 0, []
    for axis, p in enumerate(_axes(c)):
        for i in range(p):
            b = c["base"]
            if c["scaling"] == "base":
                b *= c["factor"] ** (p / (p - 1.0))
            f = b ** (-i / p)
            if c["scaling"] == "linear":
                f /= c["factor"]
            elif c["scaling"] == "ramp":
                w = min(1.0, max(0.0, (f * c["original"] / math.tau - 1.0) / (32.0 - 1.0)))
                f = (1.0 - w) * f / c["factor"] + w * f
            turns.append(pos[:, axis].double() * f)
    m = 1.0 + 0.1 * math.log(c["factor"]) if c["scaling"] == "ramp" else 1.0
    z = torch.polar(torch.full((len(pos), len(turns)), m, dtype=torch.float64, device="cuda"), torch.stack(turns, 1))
    if c["kind"] == "tables":
        return z.real.contiguous(), z.imag.contiguous()
    if c["inverse"]:
        z = z.conj()
    outs = []
    for x in (q, k):
        y = x.double()
        for i in range(len(turns)):
            a, b = (i, i + c["rotary"] // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
            t = torch.complex(x[..., a].double(), x[..., b].double()) * z[:, i, None]
            y[..., a], y[..., b] = t.real, t.imag
        outs.append(y)
    return tuple(outs)


def _exact_state(c, seed):
    """Token by token."""
    q, k, v, decay, s = _raw_state(c, seed)
    news = _ints(c["news"])
    G, D = c["q_heads"] // c["kv_heads"], c["dim"]
    s, out = s.double(), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    order = sorted(range(len(news)), key=lambda i: -news[i])
    first = [sum(news[:i]) for i in order]
    s, lens = s[order], sorted(news, reverse=True)
    at = torch.tensor(first, device="cuda")
    kept = decay.double().exp()
    for t in range(lens[0]):
        while lens[-1] <= t:                            # sequences that have ended wait behind the others
            lens.pop()
        a, b = s[: len(lens)], at[: len(lens)] + t
        a *= kept[b][..., None, None] if c["decay"] == "token" else kept[:, None, None]
        a += k[b].double()[..., :, None] * v[b].double()[..., None, :]
        out[b] = (q[b].double().unflatten(1, (-1, G)) @ a).flatten(1, 2) / math.sqrt(D)
    back = torch.empty_like(s)
    back[torch.tensor(order, device="cuda")] = s
    return out, back


def exact(case, seed):
    return _exact_state(case, seed) if case["kind"] == "state" else _exact_rotary(case, seed)
