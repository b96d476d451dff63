"""Several texts generated at once by a small decoder over a paged 8-bit cache.

    python examples/paged_generation.py [--streams 16] [--tokens 64] [--layers 4]

Prompts of different lengths enter in one step, then every step decodes a token of each stream; a stream that ends
gives its pages back and the next prompt takes its place.  Every layer's keys and queries are rotated and its keys and
values held by one launch (PagedKVCache.append), and its attention reads them (PagedKVCache.attend).  The weights are random: what is
shown is how the calls go together, and what they cost.
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import torch

from paper_2605_09681_gb300 import PagedKVCache


class Decoder:
    """A pre-norm decoder of `layers` blocks with grouped heads, bf16 weights made from `seed`."""

    def __init__(self, layers=4, q_heads=16, kv_heads=4, head_dim=64, vocab=1000, positions=8192, seed=0):
        self.layers, self.q_heads, self.kv_heads, self.head_dim, self.vocab = layers, q_heads, kv_heads, head_dim, vocab
        d = q_heads * head_dim
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda n, m, gain=1.0: (torch.randn(n, m, generator=g, device="cuda") * gain * n ** -0.5).to(torch.bfloat16)
        self.embed = torch.randn(vocab, d, generator=g, device="cuda").to(torch.bfloat16)
        self.blocks = [(w(d, (q_heads + 2 * kv_heads) * head_dim, 1.5), w(d, d), w(d, 4 * d), w(4 * d, d)) for _ in range(layers)]
        freq = 10000.0 ** (-torch.arange(0, head_dim, 2, device="cuda", dtype=torch.float32) / head_dim)
        angle = torch.arange(positions, device="cuda", dtype=torch.float32)[:, None] * freq
        self.cos, self.sin = angle.cos().contiguous(), angle.sin().contiguous()

    def cache(self, streams, tokens, page_tokens=64):
        """A cache for `streams` sequences of at most `tokens` tokens."""
        pages = streams * -(-tokens // page_tokens)
        return PagedKVCache(n_layers=self.layers, n_q_heads=self.q_heads, n_kv_heads=self.kv_heads, head_dim=self.head_dim,
                            page_tokens=page_tokens, n_pages=pages, max_seqs=streams, max_seq_tokens=tokens)

    @staticmethod
    def _norm(x):
        return torch.nn.functional.rms_norm(x.float(), (x.shape[-1],)).to(torch.bfloat16)

    def forward(self, cache, tokens, seqs, counts):
        """Logits of each sequence's last token; tokens: those of all sequences, counts[i] of seqs[i]."""
        cache.step(seqs, counts)
        Hq, Hkv, D = self.q_heads, self.kv_heads, self.head_dim
        x = self.embed[tokens]
        for layer, (wqkv, wo, w1, w2) in enumerate(self.blocks):
            qkv = (self._norm(x) @ wqkv).view(len(tokens), Hq + 2 * Hkv, D)
            Q, K, V = qkv[:, :Hq], qkv[:, Hq: Hq + Hkv], qkv[:, Hq + Hkv:]     # rows of the projection, as they lie
            Q = cache.append(layer, K, V, self.cos, self.sin, Q=Q)
            x = x + cache.attend(layer, Q).view(len(tokens), Hq * D) @ wo
            x = x + torch.nn.functional.gelu(self._norm(x) @ w1) @ w2
        last = torch.tensor(counts, device="cuda").cumsum(0) - 1
        return self._norm(x[last]) @ self.embed.T


def generate(model, cache, prompts, n_tokens, streams):
    """n_tokens more tokens (the likeliest) for each prompt, `streams` of them at a time."""
    texts = [list(p) for p in prompts]
    waiting, running = list(range(len(prompts))), {}       # running: sequence -> prompt
    free = list(range(streams))
    while waiting or running:
        batch = []                                         # (sequence, prompt, tokens of this step)
        for seq, i in running.items():
            batch.append((seq, i, texts[i][-1:]))
        while waiting and free:
            seq, i = free.pop(), waiting.pop(0)
            running[seq] = i
            batch.append((seq, i, texts[i]))
        tokens = torch.tensor([t for _, _, ts in batch for t in ts], device="cuda")
        logits = model.forward(cache, tokens, [s for s, _, _ in batch], [len(ts) for _, _, ts in batch])
        for (seq, i, _), t in zip(batch, logits.argmax(-1).tolist()):
            texts[i].append(t)
            if len(texts[i]) == len(prompts[i]) + n_tokens:
                del running[seq]
                cache.drop(seq)
                free.append(seq)
    if cache.sync_status() != 0:
        raise RuntimeError("the cache reports values that were not finite, or a wait that ran out")
    return texts


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--streams", type=int, default=16)
    ap.add_argument("--prompts", type=int, default=24)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args()
    model = Decoder(layers=a.layers)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.vocab, (int(n),), generator=g).tolist()
               for n in torch.randint(1, 1500, (a.prompts,), generator=g)]
    with model.cache(a.streams, 2048) as cache:
        generate(model, cache, prompts[:1], 2, a.streams)  # first use of the libraries
        torch.cuda.synchronize()
        t = time.perf_counter()
        texts = generate(model, cache, prompts, a.tokens, a.streams)
        t = time.perf_counter() - t
        print("%d prompts of %d to %d tokens, %d streams: %d new tokens in %.2f s, %d kernels of the cache, %.0f MB held"
              % (len(prompts), min(map(len, prompts)), max(map(len, prompts)), a.streams, len(texts) * a.tokens, t,
                 cache.launch_count(), cache.reserved_bytes() / 1e6))


if __name__ == "__main__":
    main()
