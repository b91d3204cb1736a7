"""Learns word vectors, indexes them, and answers with them.

    python -m paper_1908_10396_amd.learn [--words 20000] [--dim 64] [--steps 300] [--batch 4096] [--dtype f32]

The searched points of this library are rows that a model learned; this is such a model, small, from the first
gradient to the answers of its index. Pairs of words come from a made-up corpus, in which every word is followed by words
of its own topic. A pair's first word is looked up and normalised to a query, and the loss is minus the log
probability of the second one under the softmax over all words; queries and answers share one table:

    q = layer_norm(E[a]) w + b,    loss = -mean log softmax(c E q)[b],    c = 1 / sqrt(d)

Both gradients of the table meet in one tensor, which torch's Adam applies. Then the table is trained,
encoded and searched as any other points are, and what the search returns gets its probabilities from the same softmax.
"""
import argparse
import json
import math
import sys
import time

import torch

import paper_1908_10396_amd as avq

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Corpus:
    """Pairs (a, b) of words of one topic; a topic's words are seeded, random ones."""

    def __init__(self, words, topic=16, seed=0, device="cuda"):
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.device, self.topic = device, topic
        self.count = words // topic * topic
        self.words = torch.randperm(words, generator=self.gen, device=device)[: self.count].to(torch.int32)

    def pairs(self, count):
        a = torch.randint(self.count, (count,), generator=self.gen, device=self.device)
        b = a // self.topic * self.topic + torch.randint(self.topic, (count,), generator=self.gen, device=self.device)
        return self.words[a], self.words[b]


class Model:
    """One table of word vectors and a layer norm: kept in 32 bits for the optimiser, computed with in `dtype`."""

    def __init__(self, words, dim, dtype=torch.float32, seed=0, rate=0.02, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.table = torch.nn.Parameter(torch.randn(words, dim, generator=gen, device=device))
        self.weight = torch.nn.Parameter(torch.ones(dim, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(dim, device=device))
        self.dtype, self.scale = dtype, 1.0 / math.sqrt(dim)
        self.adam = torch.optim.Adam([self.table, self.weight, self.bias], lr=rate)

    def cast(self):
        with torch.no_grad():
            return [p.to(self.dtype) for p in (self.table, self.weight, self.bias)]

    def queries(self, words):
        table, weight, bias = self.cast()
        return avq.layer_norm(avq.embed(table, words), weight, bias)[0]

    def gradients(self, a, b):
        """Loss of the pairs (a, b) and its gradients for the table, the norm's weight and its bias."""
        table, weight, bias = self.cast()
        x = avq.embed(table, a)
        q, mean, rstd = avq.layer_norm(x, weight, bias)
        p = avq.log_probs(table, q, b, scale=self.scale)
        up = torch.full_like(p.logp, -1.0 / a.numel())
        dq, dtable = avq.log_probs_grad(table, q, b, p.lse, up, scale=self.scale)
        dx, dweight, dbias = avq.layer_norm_grad(dq, x, mean, rstd, weight)
        avq.embed_grad(dx, a, out=dtable, accumulate=True)
        return -p.logp.mean(), dtable, dweight, dbias

    def step(self, a, b):
        loss, *grads = self.gradients(a, b)
        for p, g in zip((self.table, self.weight, self.bias), grads):
            p.grad = g.to(p.dtype)
        self.adam.step()
        return loss


def index_of(model, M, bits=4, seed=0):
    """The learned table as an index of this library."""
    points = model.table.detach()
    idx = avq.Index(points.shape[1], M, bits, seed=seed)
    idx.train(points)
    idx.encode(points)
    return idx


def answer(model, idx, words, k, reorder_k):
    """The k likeliest next words by search: (ids, their log probabilities, the softmax's other results)."""
    q = model.queries(words).float()
    ids, _ = idx.search(q, k, reorder_k)
    p = idx.log_probs(q, ids, scale=model.scale)
    return ids, p.logp, p


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--words", type=int, default=20000)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--dtype", choices=sorted(DTYPES), default="f32")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()

    corpus = Corpus(args.words, seed=args.seed)
    model = Model(args.words, args.dim, DTYPES[args.dtype], seed=args.seed)
    losses = []
    for s in range(args.steps):
        a, b = corpus.pairs(args.batch)
        if s == 1:
            torch.cuda.synchronize()
            began = time.time()
        losses.append(model.step(a, b))
        if (s + 1) % 50 == 0:
            print("step %d: loss %.4f" % (s + 1, float(losses[-1])), file=sys.stderr, flush=True)
    torch.cuda.synchronize()
    ms = (time.time() - began) * 1e3 / (args.steps - 1) if args.steps > 1 else None

    idx = index_of(model, args.dim // 2)
    a, b = corpus.pairs(256)
    ids, logp, p = answer(model, idx, a, 16, 256)
    best = avq.log_probs(model.table.detach(), model.queries(a).float(), k=16, scale=model.scale)
    out = {"words": args.words, "dim": args.dim, "batch": args.batch, "dtype": args.dtype, "ms_per_step": ms,
           "loss": [float(x) for x in losses[:: max(1, args.steps // 6)]] + [float(losses[-1])] if losses else [],
           "least_possible_loss": math.log(corpus.topic), "entropy_mean": float(p.entropy.mean()),
           "probability_found": float(logp.exp().sum(1).mean()), "probability_of_the_16_best": float(best.alt_logp.exp().sum(1).mean()),
           "next_word_among_found": float((ids == b[:, None]).any(1).float().mean())}
    print(json.dumps(out), flush=True)


if __name__ == "__main__":
    main()
