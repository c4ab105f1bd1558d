"""Retrieval and generation on one GPU: search, shared passages, drafts from the
passage's own words.

A tiny causal transformer with random weights stands in for the generator and
its token embeddings' means for the retriever, so the words mean nothing; what
is real is the path of a request:

1. every passage is encoded into the index (`Index.add`) and prompted once: its
   keys and values stay in the cache as 8-bit pages (`extend`, `append`,
   `attention`);
2. a request searches the index (`Index.search`) and forks the pages of the
   passage that it found (`fork`), then adds its question behind them: the part
   of a page that the passage fills is copied, the rest is shared;
3. each step takes the words that follow the last one in the passage as drafts,
   scores them all with one attention over the cache, keeps those that the
   target's probabilities accept (`verify_drafts`) and cuts the others off
   (`truncate`).  Counts and lengths stay on the device;
4. finished requests give their pages back, and the pool is packed (`compact`).

    python examples/answer.py [--requests 4] [--steps 12] [--codes int8]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_16973_gb300 as tq  # noqa: E402

VOCAB, WIDTH, LAYERS, HEADS, KV_HEADS, DIM = 512, 256, 2, 8, 2, 64


class Model:
    """Pre-norm attention layers and a product with the embeddings; keys and values live in `cache`."""

    def __init__(self, cache, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *s: (torch.randn(*s, device="cuda", generator=g) / s[0] ** 0.5).to(torch.bfloat16)  # noqa: E731
        self.cache = cache
        self.embed = torch.randn(VOCAB, WIDTH, device="cuda", generator=g).to(torch.bfloat16)
        self.qkv = [draw(WIDTH, (HEADS + 2 * KV_HEADS) * DIM) for _ in range(LAYERS)]
        self.out = [draw(HEADS * DIM, WIDTH) for _ in range(LAYERS)]

    def __call__(self, tokens, slots, starts):
        """Probabilities behind each of the sequences' last tokens: `tokens` [total],
        those of slots[i] at starts[i] .. starts[i+1] - 1."""
        x = self.embed[tokens]
        for layer in range(LAYERS):
            rows = (torch.nn.functional.layer_norm(x, (WIDTH,)) @ self.qkv[layer]).view(len(tokens), -1, DIM)
            q, k, v = rows[:, :HEADS], rows[:, HEADS: HEADS + KV_HEADS], rows[:, HEADS + KV_HEADS:]
            self.cache.append(layer, slots, starts, k, v)
            x = x + self.cache.attention(layer, slots, starts, q).flatten(1) @ self.out[layer]
        x = torch.nn.functional.layer_norm(x, (WIDTH,)).float()
        return torch.softmax(x @ self.embed.float().t() / WIDTH ** 0.5, dim=1)


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def answer(requests=4, steps=12, drafts=3, passages=16, codes="int8", seed=0):
    """Runs the path; returns (tokens of each request, the passage each one found, the cache, words accepted per step)."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    texts = [rng.integers(0, VOCAB, int(n)) for n in rng.integers(40, 150, passages)]
    slots_all = passages + requests
    cache = tq.KVCache(pages=1024, slots=slots_all, max_pages=16, kv_heads=KV_HEADS, head_dim=DIM, page_tokens=32,
                       layers=LAYERS, codes=codes)
    model = Model(cache, seed)

    # the passages: vectors for the index, pages for the cache
    vectors = torch.stack([model.embed[torch.from_numpy(t).cuda()].float().mean(0) for t in texts])
    index = tq.Index(d=WIDTH, bits=4, capacity=passages)
    index.add(vectors.cpu().numpy())
    lengths = [len(t) for t in texts]
    own = ints(range(passages))
    cache.extend(own, ints(lengths))
    model(torch.from_numpy(np.concatenate(texts)).cuda(), own, ints(np.concatenate([[0], np.cumsum(lengths)])))

    # the requests: a question near one passage each; its pages are shared
    aim = rng.integers(0, passages, requests)
    found, _ = index.search(vectors.cpu().numpy()[aim] + rng.normal(0, 0.01, (requests, WIDTH)).astype(np.float32), k=1)
    found = found.cpu().numpy()[:, 0]
    slots = ints(range(passages, slots_all))
    cache.fork(slots, ints(found))
    question = [texts[p][:5] for p in found]  # (a question in the passage's words)
    cache.extend(slots, ints(len(t) for t in question))
    starts = ints(np.concatenate([[0], np.cumsum([len(t) for t in question])]))
    probs = model(torch.from_numpy(np.concatenate(question)).cuda(), slots, starts)
    last = probs[(starts[1:] - 1).long()].argmax(1).to(torch.int32)

    # where each passage goes on behind a word (the place of its first occurrence), for the drafts
    after = torch.zeros(requests, VOCAB, drafts, dtype=torch.int32, device="cuda")
    for i, p in enumerate(found):
        t = texts[p]
        for at in range(len(t) - drafts - 1, -1, -1):
            after[i, t[at]] = torch.from_numpy(t[at + 1: at + 1 + drafts].astype(np.int32)).cuda()
    row = torch.arange(requests, device="cuda")
    starts = ints(range(0, (drafts + 1) * requests + 1, drafts + 1))
    counts = ints([drafts + 1] * requests)
    told, accepted_words = [[] for _ in range(requests)], []
    for _ in range(steps):
        drafted = after[row, last.long()]
        held = cache.lens[slots.long()]
        cache.extend(slots, counts)
        probs = model(torch.cat([last[:, None], drafted], 1).flatten(), slots, starts).view(requests, drafts + 1, VOCAB)
        tokens, accepted = tq.verify_drafts(
            probs, drafted, torch.rand(requests, drafts, device="cuda", generator=g),
            torch.empty(requests, VOCAB, device="cuda").exponential_(generator=g).clamp_(min=1e-30))
        cache.truncate(slots, held + 1 + accepted)  # the last word and the accepted drafts stay
        last = tokens.gather(1, accepted.long()[:, None])[:, 0]
        accepted_words.append(accepted)
        for i, t in enumerate(tokens.tolist()):  # (for the reader: the loop itself needs none of it on the host)
            told[i] += [w for w in t if w >= 0]
    cache.check()
    return told, found, cache, torch.stack(accepted_words).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--codes", choices=("int8", "e4m3"), default="int8")
    a = ap.parse_args()
    told, found, cache, accepted = answer(a.requests, a.steps, codes=a.codes)
    for i, (words, passage) in enumerate(zip(told, found)):
        print(f"request {i}: passage {passage}, {len(words)} words in {a.steps} steps: {' '.join(map(str, words[:12]))} ...")
    shared = int((cache.refs > 1).sum())
    passages = cache.lens.numel() - a.requests
    cache.truncate(ints(range(passages, passages + a.requests)), ints([0] * a.requests))
    used = cache.compact()
    cache.check()
    print(f"{shared} pages were shared; {int(used)} hold the passages when the requests are gone")


if __name__ == "__main__":
    main()
