"""Learns word vectors, indexes them, and answers with them.

    python -m paper_1908_10396_amd.learn [--words 20000] [--dim 64] [--steps 300] [--batch 4096] [--dtype f32]
                                         [--sampled 0] [--student 0] [--tune preference|policy]

The searched points of this library are rows that a model learned; this is such a model, small, from the first
gradient to the answers of its index. Pairs of words come from a made-up corpus, in which every word is followed by words
of its own topic. A pair's first word is looked up and normalised to a query, and the loss is minus the log
probability of the second one under the softmax over all words; queries and answers share one table:

    q = layer_norm(E[a]) w + b,    loss = -mean log softmax(c E q)[b],    c = 1 / sqrt(d)

Both gradients of the table meet in one tensor, which torch's Adam applies. Then the table is trained,
encoded and searched as any other points are, and what the search returns gets its probabilities from the same softmax.

--sampled m learns from the softmax over the pair's word and m drawn ones instead. --student d has a second model, of d
dimensions, learn from what the first one's index returns (distillation, all other words as one answer more). --tune goes on with
walks that the model takes through its own index, word by word: of two walks from a word the one with more words of
even number is preferred (of two that have as many, neither), or it is such words that are rewarded.
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

    def forward(self, a):
        """The queries of words, and what the gradients need of how they were made."""
        table, weight, bias = self.cast()
        x = avq.embed(table, a)
        q, mean, rstd = avq.layer_norm(x, weight, bias)
        return q, (a, table, weight, x, mean, rstd)

    def backward(self, made, dq, dtable):
        """Gradients for the table, the norm's weight and its bias from those of the queries, added to the table's."""
        a, table, weight, x, mean, rstd = made
        dx, dweight, dbias = avq.layer_norm_grad(dq, x, mean, rstd, weight)
        avq.embed_grad(dx, a, out=dtable, accumulate=True)
        return dtable, dweight, dbias

    def gradients(self, a, b):
        """Loss of the pairs (a, b) and its gradients for the table, the norm's weight and its bias."""
        q, made = self.forward(a)
        table = made[1]
        p = avq.log_probs(table, q, b, scale=self.scale)
        up = torch.full_like(p.logp, -1.0 / a.numel())
        return (-p.logp.mean(),) + self.backward(made, *avq.log_probs_grad(table, q, b, p.lse, up, scale=self.scale))

    def sampled_gradients(self, a, b, drawn):
        """The same by the softmax over b and a few drawn words, drawn [pairs][m]; a drawn word that is b itself does not count."""
        q, made = self.forward(a)
        table = made[1]
        ids = torch.cat([b[:, None], drawn], 1)
        offset = torch.zeros(ids.shape, device=ids.device)
        offset[:, 1:].masked_fill_(drawn == b[:, None], -math.inf)
        p = avq.list_log_probs(table, q, ids, offset=offset, scale=self.scale)
        up = torch.zeros_like(p.logp)
        up[:, 0] = -1.0 / a.numel()
        dq, dtable, _ = avq.list_log_probs_grad(table, q, ids, p.logp, up, scale=self.scale)
        return (-p.logp[:, 0].mean(),) + self.backward(made, dq, dtable)

    def distill_gradients(self, a, ids, teacher, teacher_lse=None, temperature=1.0, listed=False):
        """Mean loss of distillation from a teacher's logits of ids [words][m], the student's probabilities being those of the softmax
        over all words, or over the list alone (`listed`, without teacher_lse: a list has all of the student's probability, and nothing is
        left for the teacher's other words)."""
        if listed and teacher_lse is not None:
            raise ValueError("teacher_lse needs the softmax over all words")
        q, made = self.forward(a)
        table, scale = made[1], self.scale / temperature
        ones = torch.full((a.numel(),), 1.0 / a.numel(), device=a.device)
        if listed:
            p = avq.list_log_probs(table, q, ids, scale=scale)
            up, loss = avq.distill_loss_grad(p.logp, teacher, ones, teacher_lse, temperature)
            dq, dtable, _ = avq.list_log_probs_grad(table, q, ids, p.logp, up, scale=scale)
        else:
            p = avq.log_probs(table, q, ids, scale=scale)
            up, loss = avq.distill_loss_grad(p.logp, teacher, ones, teacher_lse, temperature)
            dq, dtable = avq.log_probs_grad(table, q, ids, p.lse, up, scale=scale)
        return (loss.mean(),) + self.backward(made, dq, dtable)

    def _token_gradients(self, a, b, loss_of, count):
        q, made = self.forward(a)
        table = made[1]
        p = avq.log_probs(table, q, b, scale=self.scale)
        ones = torch.full((count,), 1.0 / max(count, 1), device=a.device)
        up, result = loss_of(p.logp, (b >= 0) & (b < table.shape[0]), ones)
        return (result.loss.mean(),) + self.backward(made, *avq.log_probs_grad(table, q, b, p.lse, up, scale=self.scale))

    def preference_gradients(self, a, b, offsets, ref=None, **how):
        """Mean loss of preferences between sequences of words b, each the answer to the word a beside it (-1: padding)."""
        def loss_of(logp, mask, ones):
            return avq.preference_loss_grad(logp, offsets, ones, ref=ref, mask=mask, **how)
        return self._token_gradients(a, b, loss_of, (offsets.numel() - 1) // 2)

    def policy_gradients(self, a, b, old, advantage, offsets, ref=None, **how):
        """Mean clipped loss of sequences of words b that were given with log probabilities `old`."""
        def loss_of(logp, mask, ones):
            return avq.policy_loss_grad(logp, old, advantage, offsets, ones, ref=ref, mask=mask, **how)
        return self._token_gradients(a, b, loss_of, offsets.numel() - 1)

    def log_probs(self, a, b):
        """log p of the words b, each as the answer to the word a beside it."""
        return avq.log_probs(self.cast()[0], self.queries(a), b, scale=self.scale).logp

    def apply(self, loss, *grads):
        for p, g in zip((self.table, self.weight, self.bias), grads):
            p.grad = g.to(p.dtype)
        self.adam.step()
        return loss

    def step(self, a, b):
        return self.apply(*self.gradients(a, b))


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


def taught(student, teacher, idx, a, k=16, reorder_k=256):
    """A step of a student from the k answers that the teacher's index returns, all other words being one answer more."""
    ids, logp, _ = answer(teacher, idx, a, k, reorder_k)
    return student.apply(*student.distill_gradients(a, ids, logp, torch.zeros_like(logp[:, 0])))  # (log p: lse is 0)


def walks(model, idx, a, length, gen, k=16, reorder_k=256):
    """Walks of `length` words from the words a, each word drawn among the answers to the one before: (words before, words), [count][length]."""
    before, words = [], []
    for _ in range(length):
        ids, logp, _ = answer(model, idx, a, k, reorder_k)
        before.append(a)
        a = ids.gather(1, torch.multinomial(logp.exp(), 1, generator=gen))[:, 0].contiguous()
        words.append(a)
    return torch.stack(before, 1), torch.stack(words, 1)


def compared(reward):
    """Of pairs of walks [pairs][2] those of unequal rewards: the places of their walks, a pair's better one first."""
    better = (reward[:, 1] > reward[:, 0]).long()
    even = 2 * torch.arange(reward.shape[0], device=reward.device)
    return torch.stack([even + better, even + 1 - better], 1)[reward[:, 0] != reward[:, 1]].view(-1)


def tune_on(model, how, before, words, reward, first, steps=4):
    """Steps on walks, [2 pairs][length], of which two are from one word each, with rewards [pairs][2]; first: the parameters of the reference."""
    length = words.shape[1]
    if how == "preference":
        order = compared(reward)
        if order.numel() == 0:  # (equal walks say nothing)
            return
        before, words = before[order], words[order]
    before, words = before.reshape(-1).contiguous(), words.reshape(-1).contiguous()
    offsets = torch.arange(0, words.numel() + 1, length, dtype=torch.int32, device=words.device)
    old = model.log_probs(before, words)
    now = [p.data for p in (model.table, model.weight, model.bias)]
    for p, value in zip((model.table, model.weight, model.bias), first):
        p.data = value
    ref = model.log_probs(before, words)
    for p, value in zip((model.table, model.weight, model.bias), now):
        p.data = value
    for _ in range(steps):
        if how == "preference":
            model.apply(*model.preference_gradients(before, words, offsets, ref=ref, beta=0.5, smoothing=0.1))
        else:
            advantage = (reward - reward.mean(1, keepdim=True)).view(-1).contiguous()
            model.apply(*model.policy_gradients(before, words, old, advantage, offsets, ref=ref, clip=(0.2, 0.28), kl=0.04))


def tune(model, corpus, how, rounds=4, count=256, length=6, M=None):
    """Rounds of walks through the model's index, and a few steps on them each. Gives the share of even words by round."""
    shares, first = [], [p.detach().clone() for p in (model.table, model.weight, model.bias)]
    for _ in range(rounds):
        idx = index_of(model, M or model.table.shape[1] // 2)
        a = corpus.pairs(count)[0].repeat_interleave(2)  # two walks from each word
        before, words = walks(model, idx, a, length, corpus.gen)
        idx.close()
        even = (words % 2 == 0).float()
        shares.append(float(even.mean()))
        tune_on(model, how, before, words, even.mean(1).view(-1, 2), first)
    return shares


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--words", type=int, default=20000)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--batch", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--dtype", choices=sorted(DTYPES), default="f32")
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--sampled", type=int, default=0, help="learn from so many drawn words a pair, not from all")
    ap.add_argument("--student", type=int, default=0, help="dimensions of a student that learns from the model's answers")
    ap.add_argument("--tune", choices=["preference", "policy"], help="go on with the model's own walks")
    args = ap.parse_args()

    corpus = Corpus(args.words, seed=args.seed)
    model = Model(args.words, args.dim, DTYPES[args.dtype], seed=args.seed)
    losses = []
    for s in range(args.steps):
        a, b = corpus.pairs(args.batch)
        if s == 1:
            torch.cuda.synchronize()
            began = time.time()
        if args.sampled:
            drawn = torch.randint(args.words, (args.batch, args.sampled), generator=corpus.gen, device=corpus.device, dtype=torch.int32)
            losses.append(model.apply(*model.sampled_gradients(a, b, drawn)))
        else:
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
    if args.student:
        student = Model(args.words, args.student, DTYPES[args.dtype], seed=args.seed + 1)
        taught_losses = [taught(student, model, idx, corpus.pairs(args.batch)[0]) for _ in range(args.steps)]
        ids = avq.log_probs(student.cast()[0], student.queries(a), k=16, scale=student.scale).alt_ids
        out["student"] = {"dim": args.student, "loss": [float(x) for x in taught_losses[:: max(1, args.steps // 6)]],
                          "next_word_among_its_16_best": float((ids == b[:, None]).any(1).float().mean())}
    if args.tune:
        out["even_words_by_round"] = tune(model, corpus, args.tune)
    print(json.dumps(out), flush=True)


if __name__ == "__main__":
    main()
