"""Drafted decoding of a batch over a shared prompt, on caches of fixed size.

A toy decoder of one attention layer with random weights and tied INT8
embeddings.  Every step of the batch

  drafts   n tokens per sequence from the cheap model: the decoder without its
           attention (projection by sp.dense, drawing by sp.verify without drafts)
  appends  the entries of the last token and the drafts to the own caches
  attends  with all of them to the prompt and the own entries, whose attention
           weight adds up over the steps (Cache.attend; the queries of drafts
           that are refused afterwards have counted too)
  verifies the drafts against the decoder's probabilities (sp.verify); the
           entries of those that were not kept are dropped
  evicts   when a cache has come near its capacity: the entries of the most
           weight stay, and the newest (Cache.evict)

    python examples/drafted_decode.py [--batch 64] [--steps 40] [--drafts 4]

prints what the drafts gained: tokens per step and sequence, and the time.
"""
import argparse
import sys
import time
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
from paper_2606_03026_gb300 import spikeproj as sp  # noqa: E402


class DraftedDecoder:
    def __init__(self, batch=64, prompt=2048, drafts=4, vocab=8192, width=256, Hq=8, Hkv=2, D=64, capacity=512,
                 budget=384, recent=64, temperature=0.7, seed=0, device="cuda:0"):
        assert budget + drafts + 1 <= capacity
        self.B, self.n, self.V, self.Hq, self.Hkv, self.D = batch, drafts, vocab, Hq, Hkv, D
        self.capacity, self.budget, self.recent, self.temperature = capacity, budget, recent, temperature
        self.dev = device
        self.rng = torch.Generator(device=device).manual_seed(seed)
        # INT8 rows per token, their scales: embedding and vocabulary projection in one
        self.W = torch.randint(-127, 128, (vocab, width), generator=self.rng, device=device, dtype=torch.int8)
        self.scale = torch.full((vocab,), 1 / (74 * width ** 0.5), device=device)
        self.Wqkv = self.normal(width, (Hq + 2 * Hkv) * D)
        # what follows a token, and how far the attention (a mean over many
        # entries) changes that: the drafts are often right, not always
        self.Wnext = 3 * self.normal(width, width)
        self.Wo = 10 * self.normal(Hq * D, width)
        bf16 = dict(dtype=torch.bfloat16, device=device)
        _, self.pk, self.pv = self.qkv(torch.randint(0, vocab, (prompt,), generator=self.rng, device=device))
        self.k, self.v = (torch.zeros(batch, capacity, Hkv, D, **bf16) for _ in range(2))
        # an eviction writes weights and positions to the other of two buffers
        self.weights, self.weights2 = (torch.zeros(batch, Hkv, capacity, device=device) for _ in range(2))
        self.pos, self.pos2 = (torch.zeros(batch, Hkv, capacity, dtype=torch.int32, device=device) for _ in range(2))
        self.lens, self.lens2, self.now = (torch.zeros(batch, dtype=torch.int32, device=device) for _ in range(3))
        self.last = torch.randint(0, vocab, (batch,), generator=self.rng, device=device, dtype=torch.int32)
        self.most = 0                        # entries of a sequence at most, known without asking the device
        self.cache = sp.Cache(batch, Hq, Hkv, D, capacity, max_T=drafts + 1, weights=True)

    def normal(self, rows, cols):
        return torch.randn(rows, cols, generator=self.rng, device=self.dev) * rows ** -0.5

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.rng, device=self.dev)

    def embed(self, tokens):
        return self.W[tokens.long()].float() * (1 / 74)

    def qkv(self, tokens):
        q, k, v = (self.embed(tokens) @ self.Wqkv).bfloat16().split([x * self.D for x in (self.Hq, self.Hkv, self.Hkv)], -1)
        return [x.reshape(*tokens.shape, -1, self.D) for x in (q, k, v)]

    def probabilities(self, hidden):
        """[..., width] -> [..., V]"""
        x = hidden.reshape(-1, hidden.shape[-1]).contiguous()
        z = torch.empty(x.shape[0], self.V, device=self.dev)
        for i in range(0, len(x), sp.SPIKE_PROJ_DENSE_MAX_B):
            sp.dense(self.W, self.scale, x[i:i + sp.SPIKE_PROJ_DENSE_MAX_B], z[i:i + sp.SPIKE_PROJ_DENSE_MAX_B])
        return torch.softmax(z / self.temperature, -1).reshape(*hidden.shape[:-1], self.V)

    def draw(self, p):
        """One token per row of p: a verification of no drafts."""
        token, none = (torch.empty(shape, dtype=torch.int32, device=self.dev) for shape in ((len(p), 1), (len(p),)))
        sp.verify(p.unsqueeze(1), None, None, None, self.uniform(len(p)), none, token)
        return token[:, 0]

    def step(self):
        """Up to drafts + 1 tokens per sequence: [B, drafts + 1], -1 past them."""
        B, n, i32 = self.B, self.n, dict(dtype=torch.int32, device=self.dev)
        if self.most + n + 1 > self.capacity:
            self.cache.evict(self.k, self.v, self.weights, self.pos, self.lens, self.now, self.budget, self.recent,
                             self.weights2, self.pos2, self.lens2)
            self.weights, self.weights2 = self.weights2, self.weights
            self.pos, self.pos2 = self.pos2, self.pos
            self.lens, self.lens2 = self.lens2, self.lens
            self.most = self.budget
        tokens = [self.last]
        q = torch.empty(B, n, self.V, device=self.dev)
        for t in range(n):
            q[:, t] = self.probabilities(self.embed(tokens[-1]) @ self.Wnext)
            tokens.append(self.draw(q[:, t]))
        tokens = torch.stack(tokens, 1)                          # [B, n + 1]
        # their entries: slots lens .. lens + n, no weight yet
        query, k, v = self.qkv(tokens)
        slots = self.lens.unsqueeze(1) + torch.arange(n + 1, **i32)
        seqs = torch.arange(B, device=self.dev).unsqueeze(1)
        self.k[seqs, slots], self.v[seqs, slots] = k, v
        heads = slots.long().unsqueeze(1).expand(B, self.Hkv, n + 1)
        self.weights.scatter_(2, heads, 0.0)
        self.pos.scatter_(2, heads, (self.now.unsqueeze(1) + torch.arange(n + 1, **i32)).unsqueeze(1).expand_as(heads))
        self.lens += n + 1
        out = torch.empty_like(query)
        self.cache.attend(query, self.k, self.v, self.lens, out, self.pk, self.pv, self.weights)
        p = self.probabilities(self.embed(tokens) @ self.Wnext + out.flatten(2).float() @ self.Wo)
        kept, result = torch.empty(B, **i32), torch.empty(B, n + 1, **i32)
        sp.verify(p, q, tokens[:, 1:], self.uniform(B, n), self.uniform(B), kept, result)
        # the last token and the kept drafts stay
        self.lens += kept - n
        self.now += kept + 1
        self.most = min(self.most + n + 1, self.capacity)
        self.last = result.gather(1, kept.long().unsqueeze(1))[:, 0]
        return result

    def close(self):
        assert self.cache.status() == sp.SP_OK
        self.cache.close()


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--batch", type=int, default=64)
    a.add_argument("--steps", type=int, default=40)
    a.add_argument("--drafts", type=int, default=4)
    a = a.parse_args()
    decoder = DraftedDecoder(a.batch, drafts=a.drafts)
    decoder.step()                                               # warm-up
    torch.cuda.synchronize()
    start, made = time.perf_counter(), 0
    for _ in range(a.steps):
        made += int((decoder.step() >= 0).sum())
    torch.cuda.synchronize()
    seconds = time.perf_counter() - start
    print(f"{a.batch} sequences, {a.drafts} drafts: {made / a.steps / a.batch:.2f} tokens per step and sequence, "
          f"{1e3 * seconds / a.steps:.2f} ms per step, {made / seconds:.0f} tokens/s")
    decoder.close()


if __name__ == "__main__":
    main()
