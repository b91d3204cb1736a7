"""Operators around learned vectors, as cases that can be timed.

The rows that an index holds are vectors that some model learned, one a word or a
class, and its queries are what the model makes of its input. These operators
learn and use such rows: rows are looked up by their ids (`embed`) and get their
gradient back from them (`embed_grad`); looked-up rows are normalised to queries
(`norm`, `norm_grad`); a query's inner products with all rows are its logits, whose
log probabilities, entropy and best alternatives are the answer (`probs`) and whose
gradient with respect to the queries and to all rows is what training needs (`train`).

Sizes: the rows are those of `synth_inputs.CONFIGS` (10,000 x 32, 1,183,514 x 100) and
of the paper's classification table (670,091 classes of 1,024 dimensions); batches
are anything from one request to some tens of thousands of words.
"""
import math

import torch

#: False: the plain form, in elementary torch operations. True: this framework's operators.
own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
GLOVE = dict(n=1_183_514, d=100)
WIDE = dict(n=670_091, d=1024)
EPS = 1e-5
IGNORED = 0.03  # share of ids that are padding (-1)


def listed():
    return [
        # the words of one short request, looked up: all latency
        dict(name="embed_few", kind="embed", **GLOVE, count=7, type="f32"),
        # the words of a training batch, rows of 2 KB
        dict(name="embed_batch", kind="embed", **WIDE, count=65_536, type="bf16"),
        # the gradient of a batch of words, as frequent as words are, over the whole table (odd count, rows of 400 bytes)
        dict(name="embed_grad_glove", kind="embed_grad", **GLOVE, count=50_001, type="f32"),
        # the same for a table of wide rows
        dict(name="embed_grad_wide", kind="embed_grad", **WIDE, count=131_072, type="bf16"),
        # the rows of a request normalised to queries: all latency
        dict(name="norm_few", kind="norm", count=7, d=100, type="f32"),
        # the rows of a training batch
        dict(name="norm_batch", kind="norm", count=65_536, d=1024, type="bf16"),
        # and their gradient, with that of weight and bias
        dict(name="norm_grad_batch", kind="norm_grad", count=65_536, d=1024, type="bf16"),
        # one request answered: the best ten classes with their log probabilities
        dict(name="probs_one", kind="probs", **GLOVE, count=1, k=10, given=1, type="f32"),
        # requests collected for a moment, wide rows
        dict(name="probs_some", kind="probs", **WIDE, count=24, k=20, given=1, type="bf16"),
        # an evaluation: every query's ten best and the log probabilities of three given classes
        dict(name="probs_batch", kind="probs", **GLOVE, count=2_048, k=10, given=3, type="f32"),
        # a training step of word vectors: the loss and the gradients of queries and rows (odd number of queries)
        dict(name="train_glove", kind="train", **GLOVE, count=1_001, type="f32"),
        # a training step of the classification layer
        dict(name="train_wide", kind="train", **WIDE, count=1_024, type="bf16"),
    ]


# no drawn case costs more than the largest listed ones: rows times queries times dimensions, logits, values of the rows
MOST_WORK = 0.7e12
MOST_LOGITS = 1_400_000_000
MOST_VALUES = 600_000_000


def draw(rng):
    """One more case: any kind, sizes spread over their logarithm between the listed ones' smallest and largest."""
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "probs", "train"])
    case = {"kind": kind, "type": rng.choice(["f32", "bf16", "f16"])}
    case["d"] = spread(32, 1024)
    if kind in ("norm", "norm_grad"):
        case["count"] = spread(1, 65_536)
        return case
    case["n"] = spread(10_000, min(1_183_514, MOST_VALUES // case["d"]))
    if kind in ("embed", "embed_grad"):
        case["count"] = spread(1, 65_536 if kind == "embed" else 131_072)
        return case
    most = min(2_048, int(MOST_WORK / (case["n"] * case["d"])), MOST_LOGITS // case["n"])
    case["count"] = spread(1, max(1, most // 2 if kind == "train" else most))
    if kind == "probs":
        case["k"] = rng.choice([0, 1, 5, 10, 20, 50])
        case["given"] = rng.choice([1, 1, 3, 10])
    return case


# ---- inputs ----------------------------------------------------------------------------

def _logit_scale(d):
    """A power of two that gives logits a deviation of about two for rows and queries of deviation one."""
    return 2.0 ** round(math.log2(2.0 / math.sqrt(d)))


def _ids(shape, n, gen):
    """Ids as frequent as words are (the r-th most frequent one in proportion to 1/r), some of them padding."""
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(n + 1.0)).long() - 1).clamp_(0, n - 1).int()
    return torch.where(torch.rand(shape, generator=gen, device="cuda") < IGNORED, -1, ids)


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, d, count, dtype = case["kind"], case["d"], case["count"], TYPES[case["type"]]
    state = {"case": case}
    if kind == "embed":
        state["table"] = _normal((case["n"], d), gen).to(dtype)
        state["ids"] = _ids((count,), case["n"], gen)
    elif kind == "embed_grad":
        state["grad"] = _normal((count, d), gen).to(dtype)
        state["ids"] = _ids((count,), case["n"], gen)
    elif kind in ("norm", "norm_grad"):
        # rows of unequal length and with a mean of their own, as sums of embeddings have
        x = _normal((count, d), gen) * torch.exp(0.5 * _normal((count, 1), gen)) + 0.3 * _normal((count, 1), gen)
        state["x"] = x.to(dtype)
        state["weight"] = (1.0 + 0.2 * _normal((d,), gen)).to(dtype)
        state["bias"] = (0.1 * _normal((d,), gen)).to(dtype)
        if kind == "norm_grad":
            state["grad"] = _normal((count, d), gen).to(dtype)
            x = state["x"].float()  # the forward pass left these
            state["mean"] = x.mean(1)
            state["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + EPS)
    else:
        # Where alternatives are asked for, rows and queries lie on a grid (multiples of 1/32, as vectors kept in 8 bits do),
        # so that equal logits occur and no order of additions decides which of two comes first.
        grid = kind == "probs" and case["k"] > 0

        def on(x):
            return (torch.round(x * 32.0).clamp_(-127, 127) / 32.0) if grid else x

        points = on(_normal((case["n"], d), gen)).to(dtype)
        given = case.get("given", 1)
        shape = (count,) if kind == "train" else (count, given)
        ids = _ids(shape, case["n"], gen)
        # a query has something of the row it should find, a few have much of it
        near = points[ids.reshape(count, -1)[:, 0].clamp(min=0).long()].float()
        share = 0.35 * torch.rand((count, 1), generator=gen, device="cuda")
        share = torch.where(torch.rand((count, 1), generator=gen, device="cuda") < 0.05, 0.9, share)
        queries = on(share * near + torch.sqrt(1.0 - share * share) * _normal((count, d), gen)).to(dtype)
        state.update(points=points, queries=queries, ids=ids, scale=_logit_scale(d))
        if kind == "train":
            # the loss is the mean of -log p: every query weighs the same but those left out
            state["grad_logp"] = torch.where(ids >= 0, -1.0 / count, 0.0)
    return state


# ---- one pass --------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_1908_10396_amd as avq
    case, kind = state["case"], state["case"]["kind"]
    if kind == "embed":
        return avq.embed(state["table"], state["ids"], scale=math.sqrt(case["d"]))
    if kind == "embed_grad":
        return avq.embed_grad(state["grad"], state["ids"], case["n"], scale=math.sqrt(case["d"]))
    if kind == "norm":
        y, mean, rstd = avq.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        dx, dw, db = avq.layer_norm_grad(state["grad"], state["x"], state["mean"], state["rstd"], state["weight"])
        return {"x": dx, "weight": dw, "bias": db}
    k = case.get("k", 0)
    r = avq.log_probs(state["points"], state["queries"], state["ids"], k=k, scale=state["scale"])
    out = {"logp": r.logp, "lse": r.lse, "entropy": r.entropy}
    if k:
        out["alt_ids"], out["alt_logp"] = r.alt_ids, r.alt_logp
    if kind == "train":
        out["queries"], out["points"] = avq.log_probs_grad(state["points"], state["queries"], state["ids"], r.lse,
                                                           state["grad_logp"], scale=state["scale"])
    return out


def _product_in_parts(a, b):
    """a @ b for a long inner dimension, as the sum of 64 products: one chain of a million fp32 additions would not keep
    what the inputs hold."""
    more = -a.shape[1] % 64
    a = torch.nn.functional.pad(a, (0, more)).reshape(a.shape[0], 64, -1).transpose(0, 1).contiguous()
    b = torch.nn.functional.pad(b, (0, 0, 0, more)).reshape(64, -1, b.shape[1])
    return torch.bmm(a, b).sum(0)


def _run_plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "embed":
        ids = state["ids"]
        rows = state["table"][ids.clamp(min=0).long()].float() * math.sqrt(case["d"])
        return torch.where(ids[:, None] >= 0, rows, 0.0).to(state["table"].dtype)
    if kind == "embed_grad":
        ids, grad = state["ids"], state["grad"]
        rows = torch.where(ids[:, None] >= 0, grad.float() * math.sqrt(case["d"]), 0.0)
        out = torch.zeros((case["n"], case["d"]), device="cuda")
        return out.index_add_(0, ids.clamp(min=0).long(), rows).to(grad.dtype)
    if kind == "norm":
        x = state["x"].float()
        mean = x.mean(1)
        off = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((off * off).mean(1) + EPS)
        y = off * rstd[:, None] * state["weight"].float() + state["bias"].float()
        return {"y": y.to(state["x"].dtype), "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        dy, rstd, dtype = state["grad"].float(), state["rstd"][:, None], state["x"].dtype
        xhat = (state["x"].float() - state["mean"][:, None]) * rstd
        g = dy * state["weight"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        return {"x": dx.to(dtype), "weight": (dy * xhat).sum(0).to(dtype), "bias": dy.sum(0).to(dtype)}

    points, queries, ids, scale = state["points"].float(), state["queries"].float(), state["ids"], state["scale"]
    logits = (queries @ points.t()) * scale
    top = logits.max(1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    entropy = torch.log(total)[:, 0] - (e * (logits - top)).sum(1) / total[:, 0]
    rows = ids.reshape(ids.shape[0], -1)
    logp = torch.where(rows >= 0, torch.gather(logits, 1, rows.clamp(min=0).long()) - lse[:, None], -math.inf)
    out = {"logp": logp.reshape(ids.shape), "lse": lse, "entropy": entropy}
    if case.get("k", 0):
        # the order of (logit descending, id ascending) as whole numbers, no two alike
        bits = (logits + 0.0).view(torch.int32)
        key = bits ^ ((bits >> 31) & 0x7FFFFFFF)
        key = (key.long() << 32) | (0xFFFFFFFF - torch.arange(case["n"], device="cuda"))
        best = 0xFFFFFFFF - (torch.topk(key, case["k"], dim=1).values & 0xFFFFFFFF)
        out["alt_ids"] = best.int()
        out["alt_logp"] = torch.gather(logits, 1, best) - lse[:, None]
    if case["kind"] == "train":
        weight = torch.where(ids >= 0, state["grad_logp"], 0.0)
        g = e / total * -weight[:, None]
        g.scatter_add_(1, ids.clamp(min=0).long()[:, None], weight[:, None])
        g = g * scale
        out["queries"] = _product_in_parts(g, points).to(state["queries"].dtype)
        out["points"] = (g.t() @ queries).to(state["points"].dtype)
    return out


# ---- what a pass cannot do without -------------------------------------------------------

def work(case):
    """Bytes: inputs read once, outputs written once. Flops: multiplications and additions of the definition."""
    kind, d, count, size = case["kind"], case["d"], case["count"], BYTES[case["type"]]
    if kind == "embed":  # the rows asked for, their ids, and the result
        return {"bytes": count * (2.0 * d * size + 4), "flops": 1.0 * count * d}
    if kind == "embed_grad":
        return {"bytes": count * (1.0 * d * size + 4) + 1.0 * case["n"] * d * size, "flops": 2.0 * count * d}
    if kind == "norm":
        return {"bytes": 2.0 * count * d * size + 8.0 * count + 2.0 * d * size, "flops": 8.0 * count * d}
    if kind == "norm_grad":
        return {"bytes": 3.0 * count * d * size + 8.0 * count + 3.0 * d * size, "flops": 13.0 * count * d}
    n, given, k = case["n"], case.get("given", 1), case.get("k", 0)
    rows = 1.0 * (n + count) * d * size
    small = count * (8.0 * given + 8.0 + 8.0 * k)
    if kind == "probs":
        return {"bytes": rows + small, "flops": 2.0 * n * count * d + 6.0 * n * count}
    # training: the logits once and two products of their gradient; rows and queries read, their gradients written
    return {"bytes": 2.0 * rows + small, "flops": 6.0 * n * count * d + 9.0 * n * count}


# ---- in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    kind, d, count = case["kind"], case["d"], case["count"]
    f64 = torch.float64
    if kind == "embed":
        out = torch.zeros((count, d), dtype=f64, device="cuda")
        real = torch.nonzero(state["ids"] >= 0)[:, 0]
        out[real] = state["table"].index_select(0, state["ids"][real].long()).to(f64) * math.sqrt(d)
        return out
    if kind == "embed_grad":
        out = torch.zeros((case["n"], d), dtype=f64, device="cuda")
        real = torch.nonzero(state["ids"] >= 0)[:, 0]
        out.index_put_((state["ids"][real].long(),), state["grad"][real].to(f64) * math.sqrt(d), accumulate=True)
        return out
    if kind == "norm":
        x = state["x"].to(f64)
        mean = x.sum(1) / d
        rstd = ((x.square().sum(1) / d - mean.square()) + EPS).rsqrt()
        y = (x - mean[:, None]) * rstd[:, None] * state["weight"].to(f64) + state["bias"].to(f64)
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        dy, w = state["grad"].to(f64), state["weight"].to(f64)
        xhat = (state["x"].to(f64) - state["mean"].to(f64)[:, None]) * state["rstd"].to(f64)[:, None]
        a = (dy @ w / d)[:, None]
        b = ((dy * xhat) @ w / d)[:, None]
        return {"x": (dy * w - a - xhat * b) * state["rstd"].to(f64)[:, None], "weight": (dy * xhat).sum(0), "bias": dy.sum(0)}

    n, k, ids, scale = case["n"], case.get("k", 0), state["ids"], state["scale"]
    points, queries = state["points"].to(f64), state["queries"].to(f64)
    rows = ids.reshape(count, -1).long()
    out = {"logp": torch.full(rows.shape, -math.inf, dtype=f64, device="cuda"),
           "lse": torch.empty(count, dtype=f64, device="cuda"), "entropy": torch.empty(count, dtype=f64, device="cuda")}
    if k:
        out["alt_ids"], out["alt_logp"] = None, torch.empty((count, k), dtype=f64, device="cuda")
    if kind == "train":
        out["queries"] = torch.empty((count, d), dtype=f64, device="cuda")
        out["points"] = torch.zeros((n, d), dtype=f64, device="cuda")
    step = max(1, min(count, 300_000_000 // n))
    for at in range(0, count, step):
        part = slice(at, min(count, at + step))
        q, r = queries[part], rows[part]
        logp = (q @ points.t()).mul_(scale)
        lse = torch.logsumexp(logp, 1)
        logp -= lse[:, None]
        out["lse"][part] = lse
        p = logp.exp()
        out["entropy"][part] = -(p * logp).sum(1)
        real = r >= 0
        out["logp"][part][real] = logp.gather(1, r.clamp(min=0))[real]
        if k:
            out["alt_logp"][part] = logp.topk(k, dim=1).values
        if kind == "train":
            w = torch.where(real[:, 0], state["grad_logp"][part].to(f64), 0.0)
            g = p.mul_(-w[:, None])
            line = torch.arange(q.shape[0], device="cuda")
            g[line, r[:, 0].clamp(min=0)] += w
            g *= scale
            out["queries"][part] = g @ points
            out["points"].addmm_(g.t(), q)
    out["logp"] = out["logp"].reshape(ids.shape)
    return out
