"""The paged 8-bit cache's operators as cases to be timed and compared: appending rotated keys and values, and
attention over the cache.

A case is a plain dict.  `kind` says which operator one pass is:

  append    one step's keys and values of every sequence, and its queries, are rotated, the keys and values
            rounded to E4M3 with one power-of-two scale for each page and head and appended; then what the cache
            holds is read back from the first page written on.  Outputs: the rotated queries, held K, held V.
  attend    the queries of one step over everything their sequences hold.  Output: O.

Sequences are ragged: `lens` and `news` are texts of whole numbers, one for each sequence (tokens held before
the step, tokens of the step).  The sizes are those of this repository's workloads (12 heads of 128 channels,
1560 tokens a frame, chunks of 3 frames, windows of 18) and generic ones of serving language models; `draw`
spreads the same options over the whole range.
"""
import math

import torch

own = False

_BASE = {"q_heads": 12, "kv_heads": 12, "dim": 128, "page": 64, "rope": "half", "rope_dim": 128,
         "positions": False, "causal": True, "window": 0, "sinks": 0}


def _text(values):
    return " ".join(str(int(v)) for v in values)


def _spread(n, lo, hi, step):
    """n ragged lengths from lo to hi, in an order that is not sorted."""
    return [lo + (i * step * 7919 + 13 * i) % (hi - lo + 1) for i in range(n)]


def _case(name, kind, lens, news, **kw):
    return dict(_BASE, name=name, kind=kind, lens=_text(lens), news=_text(news), **kw)


def listed():
    return [
        # the smallest append: one stream, one token (launch latency)
        _case("append_token", "append", [1560], [1]),
        # a decoding batch: 64 streams, one token each, grouped heads; pages end in each stream elsewhere
        _case("append_batch", "append", _spread(64, 1, 4095, 61), [1] * 64, q_heads=32, kv_heads=8),
        # a 480P chunk of 3 frames behind a held frame, pairs interleaved as video models rotate them, a
        # position for each token given
        _case("append_chunk", "append", [1560], [4680], page=128, rope="interleaved", positions=True),
        # ragged prompts of small heads, a part of the channels rotated
        _case("append_prompts", "append", [0, 0, 17, 0, 640, 0, 31, 0, 5], [1, 997, 2048, 333, 64, 1500, 33, 7, 2500],
              q_heads=16, kv_heads=4, dim=64, page=32, rope_dim=32),
        # the smallest attention: one token over a frame
        _case("attend_token", "attend", [1560], [1]),
        # one token over a long document: the key axis has to be split
        _case("attend_long", "attend", [131071], [1], q_heads=32, kv_heads=8),
        # a decoding batch over ragged lengths
        _case("attend_batch", "attend", _spread(64, 500, 8000, 61), [1] * 64, q_heads=32, kv_heads=8),
        # a few drafted tokens per stream to be verified, many heads over few, small heads
        _case("attend_draft", "attend", _spread(16, 200, 4000, 37), [5, 1, 8, 3] * 4, q_heads=24, kv_heads=2,
              dim=64, page=32),
        # a 480P chunk over a window of 18 frames, every query sees every key (the largest)
        _case("attend_chunk", "attend", [28080], [4680], page=128, causal=False),
        # ragged prompts, causal, grouped heads
        _case("attend_prompts", "attend", [0, 0, 129, 0, 1000, 0], [1777, 300, 2500, 4001, 512, 63], q_heads=32, kv_heads=8),
        # a long prompt's piece under a sliding window with sinks, small heads
        _case("attend_window", "attend", [14001], [2048], q_heads=16, kv_heads=4, dim=64, page=32, window=1024, sinks=4),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "attend", "attend"])
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 12])
    q = kv * rng.choice([1, 1, 2, 3, 4, 8])
    c = dict(_BASE, kind=kind, q_heads=q, kv_heads=kv, dim=dim, page=rng.choice([32, 64, 128]),
             rope=rng.choice(["half", "interleaved"]), rope_dim=dim // rng.choice([1, 1, 2]),
             positions=rng.random() < 0.3, causal=rng.random() < 0.7)
    if rng.random() < 0.25:
        c["window"] = log(64, 4096)
        c["sinks"] = rng.choice([0, 4, 100])
    for _ in range(1000):
        seqs = log(1, 64)
        style = rng.choice(["token", "few", "chunk"])
        top = {"token": 1, "few": 12, "chunk": log(16, 4680)}[style]
        news = [rng.randint(1, top) if style == "few" else max(1, int(top * rng.uniform(0.3, 1.0))) for _ in range(seqs)]
        reach = log(16, 65536 if kind == "attend" else 4096)
        lens = [rng.randint(0, reach) for _ in range(seqs)]
        c["lens"], c["news"] = _text(lens), _text(news)
        w, keys = work(c), max(a + b for a, b in zip(lens, news))
        padded = seqs * max(news) * q * keys
        if kind == "append":
            if sum(news) * (q + 2 * kv) * dim <= 4680 * 36 * 128 and sum(lens) * kv * dim <= 1 << 28:
                return c
        elif w["flops"] <= 9e11 and w["bytes"] <= 5.2e8 and padded <= 1.8e9 and seqs * keys * kv * dim <= 4e8:
            return c
    raise AssertionError("no case drawn")


# ---------------------------------------------------------------- inputs


def _ints(text):
    return [int(v) for v in text.split()]


def _normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _raw(c, seed):
    """Keys, values and queries in bf16: heads of different key scales, a few strong key channels, values whose size
    differs from token to token."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 17)
    lens, news = _ints(c["lens"]), _ints(c["news"])
    H, D = c["kv_heads"], c["dim"]
    total = sum(lens) + sum(news)
    chan = 1.0 + 5.0 * (torch.rand((H, D), generator=g, device="cuda") < 0.04)
    head = 0.5 + torch.rand((H, 1), generator=g, device="cuda")
    K = (_normal((total, H, D), g) * (chan * head)).to(torch.bfloat16)
    V = (_normal((total, H, D), g) * torch.exp(0.5 * _normal((total, 1, 1), g))).to(torch.bfloat16)
    Q = _normal((sum(news), c["q_heads"], D), g, torch.bfloat16)
    held, new, at = [], [], 0                        # tokens of a sequence: those held, then those of the step
    for a, b in zip(lens, news):
        held += range(at, at + a)
        new += range(at + a, at + a + b)
        at += a + b
    return K, V, Q, torch.tensor(held, dtype=torch.int64, device="cuda"), torch.tensor(new, dtype=torch.int64, device="cuda")


def _tables(c):
    """cos and sin [rows][rope_dim / 2] in fp32, and for each token of the step its row."""
    lens, news = _ints(c["lens"]), _ints(c["news"])
    rows = max(a + b for a, b in zip(lens, news)) + 64
    freq = 10000.0 ** (-torch.arange(0, c["rope_dim"], 2, dtype=torch.float64) / c["rope_dim"])
    ang = torch.arange(rows, dtype=torch.float64)[:, None] * freq
    shift = 37 if c["positions"] else 0              # given positions differ from the tokens' own
    pos = [a + i + shift for a, b in zip(lens, news) for i in range(b)]
    old = [i + shift for a in lens for i in range(a)]
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return ang.cos().float().cuda(), ang.sin().float().cuda(), dev(pos), dev(old)


def prepare(case, seed):
    c = case
    lens, news = _ints(c["lens"]), _ints(c["news"])
    K, V, Q, held, new = _raw(c, seed)
    append = c["kind"] == "append"
    st = {"case": c, "Q": Q}
    if append:
        cos, sin, pos, old = _tables(c)
        st |= {"K": K[new], "V": V[new], "cos": cos, "sin": sin, "pos": pos}
    if own:
        from paper_2605_09681_gb300 import PagedKVCache

        P = c["page"]
        cache = PagedKVCache(n_layers=1, n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["dim"],
                             page_tokens=P, n_pages=sum(-(-(a + b) // P) for a, b in zip(lens, news)),
                             max_seqs=len(lens), max_seq_tokens=max(a + b for a, b in zip(lens, news)), rope=c["rope"])
        seqs = list(range(len(lens)))
        if append:
            if sum(lens):
                cache.step(seqs, lens)
                cache.append(0, K[held], V[held], st["cos"], st["sin"], old if c["positions"] else None)
            cache.step(seqs, news)
        else:
            cache.step(seqs, [a + b for a, b in zip(lens, news)], n_query=news)
            cache.append(0, K, V)
        torch.cuda.synchronize()
        st["cache"] = cache
    elif append:
        st |= _plain_append_state(c, K, V, held, cos, sin, old)
    else:
        st |= _plain_attend_state(c, K, V)
    return st


# ---------------------------------------------------------------- the plain form


def _rotate(x, cos, sin, style):
    """x [tokens][heads][D] in fp32, cos and sin [tokens][R / 2]: the first R channels rotated."""
    R = 2 * cos.shape[1]
    c, s = cos[:, None, :], sin[:, None, :]
    a, b = (x[..., : R // 2], x[..., R // 2: R]) if style == "half" else (x[..., 0:R:2], x[..., 1:R:2])
    u, v = a * c - b * s, b * c + a * s
    y = torch.cat([u, v], -1) if style == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([y, x[..., R:]], -1) if R < x.shape[-1] else y


def _quantize(blocks):
    """blocks [n][page][heads][D] in fp32 -> E4M3 codes, and the exponent of each block and head [n][1][heads][1]."""
    m, e = torch.frexp(blocks.abs().amax((1, 3), keepdim=True))
    e = torch.clamp(e - 9 + (m > 0.875), -120, 120)
    return torch.ldexp(blocks, -e).to(torch.float8_e4m3fn), e


def _page_rows(first, last, page, base):
    """For each page of tokens first .. last - 1 of a sequence (first: a page's first token) the places of its
    tokens in an array in which token `first` is at `base`; -1 past the end."""
    return [[base + t - first if t < last else -1 for t in range(p, p + page)] for p in range(first, last, page)]


def _plain_append_state(c, K, V, held, cos, sin, old):
    """The open page's tokens (rotated keys in fp32, values) of each sequence, and where each page written finds its tokens
    among [open pages' | new ones]."""
    lens, news, P = _ints(c["lens"]), _ints(c["news"]), c["page"]
    keep, order, at = [], [], 0
    for a in lens:
        keep += range(at + a - a % P, at + a)
        at += a
    keep = torch.tensor(keep, dtype=torch.int64, device="cuda")
    n_keep, i, j = len(keep), 0, 0
    rows = []
    for a, b in zip(lens, news):
        mine = list(range(i, i + a % P)) + list(range(n_keep + j, n_keep + j + b))
        order += mine
        rows += _page_rows(a - a % P, a + b, P, len(order) - len(mine))
        i, j = i + a % P, j + b
    src = torch.tensor(order, dtype=torch.int64)
    rows = torch.tensor(rows, dtype=torch.int64)
    flat = rows.flatten()
    at = torch.nonzero(flat >= 0).flatten()
    tail = held[keep]
    o = old[keep].long()
    return {"tail_k": _rotate(K[tail].float(), cos[o], sin[o], c["rope"]), "tail_v": V[tail].float(),
            "rows": torch.where(rows >= 0, src[rows.clamp(min=0)], -1).cuda(), "valid": at.cuda()}


def _plain_append(st):
    c = st["case"]
    p = st["pos"].long()
    cos, sin = st["cos"][p], st["sin"][p]
    Qr = _rotate(st["Q"].float(), cos, sin, c["rope"]).to(torch.bfloat16)
    out = [Qr]
    new = (_rotate(st["K"].float(), cos, sin, c["rope"]), st["V"].float())
    for tail, x in ((st["tail_k"], new[0]), (st["tail_v"], new[1])):
        rows = st["rows"]
        blocks = torch.cat([tail, x])[rows.clamp(min=0)] * (rows >= 0)[:, :, None, None]
        codes, e = _quantize(blocks)
        values = torch.ldexp(codes.float(), e).to(torch.bfloat16)
        out.append(values.flatten(0, 1)[st["valid"]])
    return tuple(out)


def _plain_attend_state(c, K, V):
    """Pools of pages (codes, exponents), the page table, and each query's place in a padded batch."""
    lens, news, P = _ints(c["lens"]), _ints(c["news"]), c["page"]
    rows, table, at = [], [], 0
    for a, b in zip(lens, news):
        mine = _page_rows(0, a + b, P, at)
        table.append(list(range(len(rows), len(rows) + len(mine))))
        rows += mine
        at += a + b
    rows = torch.tensor(rows, dtype=torch.int64, device="cuda")
    st = {}
    for name, x in (("k", K), ("v", V)):
        codes, e = _quantize(x.float()[rows.clamp(min=0)] * (rows >= 0)[:, :, None, None])
        st[name], st[name + "_exp"] = codes, e.to(torch.int8)
    most = max(len(t) for t in table)
    st["table"] = torch.tensor([t + [0] * (most - len(t)) for t in table], dtype=torch.int64, device="cuda")
    st["keys"] = torch.tensor([a + b for a, b in zip(lens, news)], device="cuda")
    st["news"] = torch.tensor(news, device="cuda")
    st["batch"] = torch.tensor([s for s, b in enumerate(news) for _ in range(b)], device="cuda")
    st["place"] = torch.tensor([i for b in news for i in range(b)], device="cuda")
    return st


def _plain_attend(st):
    c = st["case"]
    B, H, G, D = len(st["table"]), c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    k, v = (torch.ldexp(st[n][st["table"]].float(), st[n + "_exp"][st["table"]].int()).flatten(1, 2).transpose(1, 2) for n in "kv")
    n, most = k.shape[2], max(_ints(c["news"]))
    q = torch.zeros((B, most, H, G, D), dtype=torch.float32, device="cuda")
    q[st["batch"], st["place"]] = st["Q"].float().unflatten(1, (H, G))
    q = q.permute(0, 2, 3, 1, 4).flatten(2, 3)                           # [B][H][G most][D]
    s = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).unflatten(2, (G, most))
    j = torch.arange(n, device="cuda")[None, None, :]
    end = st["keys"][:, None, None]
    pos = (st["keys"] - st["news"])[:, None, None] + torch.arange(most, device="cuda")[None, :, None]
    see = j < torch.minimum(end, pos + 1) if c["causal"] else (j < end).expand(B, most, n)
    if c["window"]:
        see = see & ((j > pos - c["window"]) | (j < c["sinks"]))
    s.masked_fill_(~see[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).unflatten(2, (G, most)) / torch.where(total > 0, total, 1.0)
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[st["batch"], st["place"]].to(torch.bfloat16)


def run(state):
    c = state["case"]
    if not own:
        return _plain_append(state) if c["kind"] == "append" else _plain_attend(state)
    cache = state["cache"]
    if c["kind"] == "append":
        Qr = cache.append(0, state["K"], state["V"], state["cos"], state["sin"], state["pos"] if c["positions"] else None, Q=state["Q"])
        return (Qr,) + cache.read(0)
    return cache.attend(0, state["Q"], causal=c["causal"], window=c["window"], sinks=c["sinks"])


# ---------------------------------------------------------------- what a pass cannot do without


def _pairs(c):
    """Visible (query, key) pairs of one query head, and keys that some query of a sequence sees, over all sequences."""
    pairs = keys = 0
    for a, b in zip(_ints(c["lens"]), _ints(c["news"])):
        n, w, k = a + b, c["window"], c["sinks"]
        lo = max(0, a - w + 1) if w else 0
        keys += n - lo + min(k if w else 0, lo)
        if not w:
            pairs += a * b + b * (b + 1) // 2 if c["causal"] else n * b
        else:
            for p in range(a, n):
                first = max(0, p - w + 1)
                pairs += (p + 1 if c["causal"] else n) - first + min(k, first)
    return pairs, keys


def work(case):
    c = case
    lens, news, P, D = _ints(c["lens"]), _ints(c["news"]), c["page"], c["dim"]
    T = sum(news)
    if c["kind"] == "append":
        held = T + sum(a % P for a in lens)          # tokens of the pages written
        row = c["kv_heads"] * D
        # K, V and Q read, the tables' rows, rotated Q and codes written; codes read and values written by the read-back
        b = T * (2 * row * 2 + 2 * c["q_heads"] * D * 2 + 4 * c["rope_dim"] + 2 * row) + held * 2 * row * 3
        f = T * (c["q_heads"] + c["kv_heads"]) * c["rope_dim"] * 3 + T * 2 * row * 2 + held * 2 * row
        return {"bytes": b, "flops": f}
    pairs, keys = _pairs(c)
    return {"bytes": 2 * T * c["q_heads"] * D * 2 + keys * c["kv_heads"] * D * 2, "flops": 4 * D * pairs * c["q_heads"]}


# ---------------------------------------------------------------- the definition in 64 bits


def _e4m3_exact(x):
    """The nearest E4M3 values of x (|x| <= 448), ties to even, in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _held_exact(x, page):
    """x [tokens][heads][D] of one sequence from a page's first token on, as the cache holds it."""
    out = torch.empty_like(x)
    for p in range(0, len(x), page):
        b = x[p: p + page]
        top = b.abs().amax((0, 2), keepdim=True)
        e = torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -120)))
        scale = torch.exp2(e)
        out[p: p + page] = _e4m3_exact(b / scale) * scale
    return out


def exact(case, seed):
    c = case
    lens, news, P, D = _ints(c["lens"]), _ints(c["news"]), c["page"], c["dim"]
    H, G = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    K, V, Q, _, _ = _raw(c, seed)
    Q = Q.double()

    def turned(x, rows):
        cos, sin, _, _ = tables
        R = c["rope_dim"]
        z = x.clone()
        for i in range(R // 2):
            u, w = (i, i + R // 2) if c["rope"] == "half" else (2 * i, 2 * i + 1)
            co, si = cos[rows, i].double()[:, None], sin[rows, i].double()[:, None]
            z[..., u] = x[..., u] * co - x[..., w] * si
            z[..., w] = x[..., u] * si + x[..., w] * co
        return z

    if c["kind"] == "append":
        tables = _tables(c)
        shift = 37 if c["positions"] else 0
        qs, ks, vs, at, qat = [], [], [], 0, 0
        for a, b in zip(lens, news):
            first = a - a % P
            rows = torch.arange(first, a + b, device="cuda") + shift
            ks.append(_held_exact(turned(K[at + first: at + a + b].double(), rows), P))
            vs.append(_held_exact(V[at + first: at + a + b].double(), P))
            qs.append(turned(Q[qat: qat + b], rows[a - first:]))
            at, qat = at + a + b, qat + b
        return torch.cat(qs), torch.cat(ks), torch.cat(vs)
    outs, at, qat = [], 0, 0
    for a, b in zip(lens, news):
        n = a + b
        k, v = _held_exact(K[at: at + n].double(), P), _held_exact(V[at: at + n].double(), P)
        o = torch.zeros((b, c["q_heads"], D), dtype=torch.float64, device="cuda")
        pos = torch.arange(a, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None, :]
        hide = torch.zeros((b, n), dtype=torch.bool, device="cuda")
        if c["causal"]:
            hide |= j > pos
        if c["window"]:
            hide |= (j <= pos - c["window"]) & (j >= c["sinks"])
        for h in range(c["q_heads"]):
            x = Q[qat: qat + b, h] @ k[:, h // G].T / math.sqrt(D)
            w = torch.softmax(x.masked_fill(hide, -math.inf), -1)
            o[:, h] = w @ v[:, h // G]
        outs.append(o)
        at, qat = at + n, qat + b
    return torch.cat(outs)
