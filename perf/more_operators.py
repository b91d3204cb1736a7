"""What learned vectors learn from, as cases that can be timed.

A table of vectors is trained on more than the softmax over all of its rows. It learns
from the rows that a search returned or a sampler drew, by a softmax over each query's
own list (`list`, `list_train`); from a larger teacher's best answers (`distill`,
`distill_train`); from pairs of answers of which one is preferred (`preference`); and from
answers that it gave itself and got a reward for (`policy`). The last three take log
probabilities and give the gradient with respect to them.

Sizes: the rows are those of `synth_inputs.CONFIGS` (1,183,514 x 100) and of the paper's
classification table (670,091 classes of 1,024 dimensions); lists are what a search
returns or a batch samples; sequences are anything from a few tokens to some thousands.
"""
import math

import numpy as np
import torch

#: False: the plain form, in elementary torch operations. True: this framework's operators.
own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
GLOVE = dict(n=1_183_514, d=100)
WIDE = dict(n=670_091, d=1024)
LEAST_REST = 2.0 ** -20  # what a student has beside the list, at least
BETA, MARGIN, SMOOTHING = 0.1, 0.05, 0.1
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04


def listed():
    return [
        # the answer of one search, as probabilities among what it returned: all latency
        dict(name="list_few", kind="list", **GLOVE, count=1, m=100, offset=False, type="f32"),
        # an evaluation: two hundred retrieved classes for every query, rows of 2 KB
        dict(name="list_batch", kind="list", **WIDE, count=2_047, m=200, offset=False, type="bf16"),
        # a step of word vectors against sampled negatives, corrected by how likely each was to be drawn (odd lists)
        dict(name="list_train_glove", kind="list_train", **GLOVE, count=2_048, m=127, offset=True, type="f32"),
        # a step of a classification layer against retrieved classes
        dict(name="list_train_wide", kind="list_train", **WIDE, count=1_024, m=64, offset=False, type="bf16"),
        # a few queries with long lists
        dict(name="list_train_long", kind="list_train", **GLOVE, count=3, m=4_000, offset=True, type="f32"),
        # a small step from a teacher's ten best: all latency
        dict(name="distill_few", kind="distill_train", count=8, m=10, rest=False, temperature=1.0, type="f32"),
        # a large batch from stored logits of 16 bits, the teacher's remaining mass as one more answer
        dict(name="distill_batch", kind="distill_train", count=65_536, m=64, rest=True, temperature=2.0, type="bf16"),
        # an evaluation against long lists (odd number of queries)
        dict(name="distill_long", kind="distill", count=8_191, m=1_000, rest=True, temperature=1.0, type="f32"),
        # a handful of short answers compared: all latency
        dict(name="preference_few", kind="preference", count=4, longest=64, average=False, reference=True),
        # a batch of pairs of answers
        dict(name="preference_batch", kind="preference", count=1_024, longest=1_024, average=False, reference=True),
        # a handful of sampled answers with their rewards
        dict(name="policy_few", kind="policy", count=8, longest=64, average=True, reference=True, each=False),
        # a batch of them, some much longer than others, an advantage for every token
        dict(name="policy_batch", kind="policy", count=512, longest=4_096, average=True, reference=True, each=True),
    ]


# no drawn case costs more than the largest listed ones
MOST_GATHERED = {"list": 2_047 * 200 * 1024, "list_train": 1_024 * 64 * 1024}  # values of the listed rows
MOST_LISTED = 1_000_000  # entries of all lists
MOST_VALUES = 600_000_000  # of a table
MOST_ELEMENTS = 8_000_000
MOST_TOKENS = 1_000_000


def draw(rng):
    """One more case: any kind, sizes spread over their logarithm between the listed ones' smallest and largest."""
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["list", "list_train", "list_train", "distill", "distill_train", "preference", "policy"])
    case = {"kind": kind}
    if kind in ("list", "list_train"):
        case["type"] = rng.choice(["f32", "bf16", "f16"])
        case["d"] = spread(32, 1024)
        case["n"] = spread(10_000, min(1_183_514, MOST_VALUES // case["d"]))
        case["m"] = spread(1, 4_096)
        case["count"] = spread(1, max(1, min(65_536, MOST_GATHERED[kind] // (case["m"] * case["d"]), MOST_LISTED // case["m"])))
        case["offset"] = rng.random() < 0.5
    elif kind in ("distill", "distill_train"):
        case["type"] = rng.choice(["f32", "bf16", "f16"])
        case["m"] = spread(1, 4_096)
        case["count"] = spread(1, max(1, min(65_536, MOST_ELEMENTS // case["m"])))
        case["rest"] = rng.random() < 0.5
        case["temperature"] = rng.choice([1.0, 1.5, 2.0, 4.0])
    else:
        case["longest"] = spread(1, 16_384)
        sequences = 2 if kind == "preference" else 1
        case["count"] = spread(1, max(1, min(8_192, MOST_TOKENS // (case["longest"] * sequences))))
        case["average"] = rng.random() < 0.5
        case["reference"] = rng.random() < 0.75
        if kind == "policy":
            case["each"] = rng.random() < 0.5
    return case


# ---- inputs ----------------------------------------------------------------------------

def _logit_scale(d):
    """A power of two that gives logits a deviation of about two for rows and queries of deviation one."""
    return 2.0 ** round(math.log2(2.0 / math.sqrt(d)))


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _uniform(shape, gen):
    return torch.rand(shape, generator=gen, device="cuda")


def _ids(shape, n, gen):
    """Ids as frequent as words are: the r-th most frequent one in proportion to 1/r, nearly."""
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(n + 1.0)).long() - 1).clamp_(0, n - 1).int()


def _lengths(count, longest, gen):
    """Four of five rows are full, the others end anywhere, some at once."""
    short = (_uniform((count,), gen) * (longest + 1)).long().clamp(max=longest)
    return torch.where(_uniform((count,), gen) < 0.8, longest, short)


def _prepare_list(case, gen, state):
    n, d, count, m, dtype = case["n"], case["d"], case["count"], case["m"], TYPES[case["type"]]
    points = _normal((n, d), gen).to(dtype)
    drawn = _ids((count, m), n, gen)
    ids = torch.where(torch.arange(m, device="cuda")[None] < _lengths(count, m, gen)[:, None], drawn, -1)
    # a query has something of the first row of its list, a few have much of it
    share = 0.35 * _uniform((count, 1), gen)
    share = torch.where(_uniform((count, 1), gen) < 0.05, 0.9, share)
    queries = (share * points[drawn[:, 0].long()].float() + torch.sqrt(1.0 - share * share) * _normal((count, d), gen)).to(dtype)
    state.update(points=points, queries=queries, ids=ids, scale=_logit_scale(d), offset=None)
    if case["offset"]:  # minus the log of how likely each was to be drawn, relative to the mean
        state["offset"] = torch.log((drawn.float() + 1.5) * (math.log(n + 1.0) / n))
    if case["kind"] == "list_train":
        # the loss is the mean of -log p of the first entry, or of a distribution over the list (every other query)
        weight = torch.softmax(2.0 * _normal((count, m), gen), 1)
        first = torch.zeros((count, m), device="cuda")
        first[:, 0] = 1.0
        odd = (torch.arange(count, device="cuda") % 2 == 1)[:, None]
        state["grad_logp"] = -torch.where(odd, weight, first) / count


def _prepare_distill(case, gen, state):
    count, m, dtype = case["count"], case["m"], TYPES[case["type"]]
    z = (3.0 * _normal((count, m), gen)).sort(1, descending=True).values.to(dtype)
    there = torch.arange(m, device="cuda")[None] < _lengths(count, m, gen)[:, None]
    t = z.double() / case["temperature"]
    # what the teacher, and the student, gave to other rows
    other = torch.log1p(0.01 + 0.5 * _uniform((2, count, 1), gen).double() ** 2)
    state["teacher"] = torch.where(there, z.float(), -math.inf).to(dtype)
    state["teacher_lse"] = (torch.logsumexp(t, 1) + other[0, :, 0]).float() if case["rest"] else None
    s = t + 0.5 * _normal((count, m), gen).double() * _uniform((count, 1), gen).double()
    state["logp"] = torch.where(there, (s - torch.logsumexp(s, 1, keepdim=True) - other[1]).float(), -math.inf)
    state["temperature"] = case["temperature"]
    state["grad_loss"] = torch.full((count,), 1.0 / count, device="cuda")


def _token_lengths(case):
    """Lengths of the sequences: spread over their logarithm, so that most are much shorter than the longest."""
    sequences = case["count"] * (2 if case["kind"] == "preference" else 1)
    return [max(1, int((case["longest"] + 0.99) ** ((i + 1.0) / sequences))) for i in range(sequences)]


def _prepare_tokens(case, gen, state):
    count, longest, kind = case["count"], case["longest"], case["kind"]
    sequences = 2 * count if kind == "preference" else count
    lengths = _token_lengths(case)
    tokens = (sum(lengths) + 63) // 64 * 64  # the batch is padded behind its last sequence
    lengths = torch.tensor(lengths, device="cuda")[torch.randperm(sequences, generator=gen, device="cuda")]
    offsets = torch.zeros(sequences + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = lengths.cumsum(0)
    mask = _uniform((tokens,), gen) >= 0.1
    logp = -2.0 * _normal((tokens,), gen).abs()
    # what log_probs gives for tokens that are no answer
    state.update(offsets=offsets, mask=mask, logp=torch.where(mask, logp, -math.inf), ref=None)
    if case["reference"]:
        state["ref"] = torch.where(mask, logp + 0.1 * _normal((tokens,), gen), -math.inf)
    if kind == "policy":
        state["old"] = torch.where(mask, logp + 0.15 * _normal((tokens,), gen), -math.inf)
        state["advantage"] = _normal((tokens,) if case["each"] else (sequences,), gen)
    state["grad_loss"] = torch.full((count,), 1.0 / count, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = {"case": case}
    if case["kind"] in ("list", "list_train"):
        _prepare_list(case, gen, state)
    elif case["kind"] in ("distill", "distill_train"):
        _prepare_distill(case, gen, state)
    else:
        _prepare_tokens(case, gen, state)
    return state


# ---- one pass --------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_1908_10396_amd as avq
    case, kind = state["case"], state["case"]["kind"]
    if kind in ("list", "list_train"):
        r = avq.list_log_probs(state["points"], state["queries"], state["ids"], offset=state["offset"], scale=state["scale"])
        out = {"logp": r.logp, "lse": r.lse}
        if kind == "list_train":
            dq, dx, do = avq.list_log_probs_grad(state["points"], state["queries"], state["ids"], r.logp, state["grad_logp"], scale=state["scale"])
            out.update(queries=dq, points=dx, offset=do)
        return out
    if kind == "distill":
        return avq.distill_loss(state["logp"], state["teacher"], state["teacher_lse"], temperature=state["temperature"])
    if kind == "distill_train":
        grad, loss = avq.distill_loss_grad(state["logp"], state["teacher"], state["grad_loss"], state["teacher_lse"], temperature=state["temperature"])
        return {"loss": loss, "grad": grad}
    if kind == "preference":
        grad, r = avq.preference_loss_grad(state["logp"], state["offsets"], state["grad_loss"], ref=state["ref"], mask=state["mask"], beta=BETA,
                                           margin=MARGIN, smoothing=SMOOTHING, average=case["average"])
        return {"loss": r.loss, "logit": r.logit, "reward": r.reward, "grad": grad}
    grad, r = avq.policy_loss_grad(state["logp"], state["old"], state["advantage"], state["offsets"], state["grad_loss"], ref=state["ref"], mask=state["mask"],
                                   clip=(CLIP_LOW, CLIP_HIGH), kl=KL if case["reference"] else 0.0, average=case["average"])
    return {"loss": r.loss, "kl": r.kl, "clipped": r.clipped, "grad": grad}


def _plain_list(state):
    points, ids, queries = state["points"], state["ids"], state["queries"].float()
    real = ids >= 0
    rows = points[ids.clamp(min=0).long()].float()
    scores = (rows * queries[:, None, :]).sum(2) * state["scale"]
    if state["offset"] is not None:
        scores = scores + state["offset"]
    scores = torch.where(real, scores, -math.inf)
    top = scores.max(1, keepdim=True).values
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(scores - top)
    total = e.sum(1, keepdim=True)
    logp = scores - top - torch.log(total)
    logp = torch.where(real, logp, -math.inf)
    out = {"logp": logp, "lse": (top + torch.log(total))[:, 0]}
    if state["case"]["kind"] == "list_train":
        g = torch.where(real, state["grad_logp"], 0.0)
        p = torch.where(real, e / total, 0.0)
        g = g - p * g.sum(1, keepdim=True)
        out["offset"] = g
        weighted = g[:, :, None] * state["scale"]
        out["queries"] = (rows * weighted).sum(1).to(points.dtype)
        into = torch.zeros(points.shape, device="cuda")
        into.index_add_(0, ids.clamp(min=0).long().reshape(-1), (weighted * queries[:, None, :]).reshape(-1, points.shape[1]))
        out["points"] = into.to(points.dtype)
    return out


def _plain_distill(state):
    # in 64 bits: where the two agree, the loss is what is left of terms that are much larger
    z, there = state["teacher"].double() / state["temperature"], state["teacher"] > -math.inf
    z = torch.where(there, z, -math.inf)
    logp = torch.where(there, state["logp"].double(), -math.inf)
    some = there.any(1)
    if state["teacher_lse"] is None:
        top = torch.where(some, z.max(1).values, 0.0)[:, None]
        lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    else:
        lse = state["teacher_lse"].double()[:, None]
    p = torch.where(there, torch.exp(z - lse), 0.0)
    loss = torch.where(there, p * (z - lse - logp), 0.0).sum(1)
    grad = -p
    if state["teacher_lse"] is not None:
        student = torch.exp(logp)
        rest = (1.0 - p.sum(1)).clamp(min=0.0)
        left = 1.0 - student.sum(1)
        mine = left.clamp(min=LEAST_REST)
        loss = loss + torch.where(rest > 0, rest * torch.log(torch.where(rest > 0, rest, 1.0) / mine), 0.0)
        grad = grad + torch.where(left > LEAST_REST, rest / mine, 0.0)[:, None] * student
    loss = torch.where(some, loss, 0.0).float()
    if state["case"]["kind"] == "distill":
        return loss
    grad = torch.where(there & some[:, None], grad, 0.0) * state["grad_loss"].double()[:, None]
    return {"loss": loss, "grad": grad.float()}


def _plain_segments(state):
    """Each token's sequence, whether it counts, and a sum over the sequences' tokens."""
    offsets, mask = state["offsets"].long(), state["mask"]
    at = torch.arange(mask.shape[0], device="cuda")
    sequences = offsets.shape[0] - 1
    which = torch.searchsorted(offsets, at, right=True) - 1
    counted = mask & (which >= 0) & (which < sequences)
    which = which.clamp(0, sequences - 1)

    def total(v):
        # in 64 bits, as differences of running sums
        running = torch.nn.functional.pad(torch.cumsum(torch.where(counted, v, 0.0), 0), (1, 0))
        return running[offsets[1:]] - running[offsets[:-1]]

    return which, counted, total


def _plain_preference(state):
    case = state["case"]
    which, counted, total = _plain_segments(state)
    ratio = state["logp"].double()
    if state["ref"] is not None:
        ratio = ratio - state["ref"].double()
    d, share = total(ratio), 1.0
    if case["average"]:
        share = 1.0 / total(torch.ones_like(ratio)).clamp(min=1.0)
        d = d * share
    reward = BETA * d
    x = reward[0::2] - reward[1::2] - MARGIN
    small = torch.exp(-x.abs())
    minus = torch.log1p(small) + (-x).clamp(min=0.0)  # -log sigma(x)
    plus = torch.log1p(small) + x.clamp(min=0.0)      # -log sigma(-x)
    loss = (1.0 - SMOOTHING) * minus + SMOOTHING * plus
    up = state["grad_loss"].double() * (SMOOTHING / (1.0 + torch.exp(-x)) - (1.0 - SMOOTHING) / (1.0 + torch.exp(x))) * BETA
    each = torch.stack([up, -up], 1).reshape(-1) * share
    return {"loss": loss.float(), "logit": x.float(), "reward": reward.float(), "grad": torch.where(counted, each[which], 0.0).float()}


def _plain_policy(state):
    case = state["case"]
    which, counted, total = _plain_segments(state)
    logp = torch.where(counted, state["logp"], 0.0).double()
    old = torch.where(counted, state["old"], 0.0).double()
    a = state["advantage"].double()
    if not case["each"]:
        a = a[which]
    ratio = torch.exp(logp - old)
    over = ((a > 0) & (ratio > 1.0 + CLIP_HIGH)) | ((a < 0) & (ratio < 1.0 - CLIP_LOW))
    held = torch.where(a > 0, 1.0 + CLIP_HIGH, 1.0 - CLIP_LOW)
    loss = -torch.where(over, held, ratio) * a
    grad = -torch.where(over, 0.0, ratio) * a
    kl = torch.zeros_like(loss)
    if case["reference"]:
        away = torch.where(counted, state["ref"], 0.0).double() - logp
        kl = torch.exp(away) - away - 1.0
        loss = loss + KL * kl
        grad = grad + KL * (1.0 - torch.exp(away))
    count = total(torch.ones_like(loss)).clamp(min=1.0)
    share = 1.0 / count if case["average"] else torch.ones_like(count)
    up = state["grad_loss"].double() * share
    return {"loss": (total(loss) * share).float(), "kl": (total(kl) * share).float(), "clipped": (total(over.double()) / count).float(),
            "grad": torch.where(counted, grad * up[which], 0.0).float()}


def _run_plain(state):
    kind = state["case"]["kind"]
    if kind in ("list", "list_train"):
        return _plain_list(state)
    if kind in ("distill", "distill_train"):
        return _plain_distill(state)
    return _plain_preference(state) if kind == "preference" else _plain_policy(state)


# ---- what a pass cannot do without -------------------------------------------------------

def _different_rows(n, drawn):
    """How many rows of the table `drawn` ids name, each at least once."""
    r = np.arange(n, dtype=np.float64)
    return float((1.0 - np.exp(-drawn * np.log((r + 2.0) / (r + 1.0)) / math.log(n + 1.0))).sum())


def work(case):
    """Bytes: inputs read once, outputs written once. Flops: multiplications and additions of the definition."""
    kind = case["kind"]
    if kind in ("list", "list_train"):
        n, d, count, size = case["n"], case["d"], case["count"], BYTES[case["type"]]
        entries = 1.0 * count * case["m"]
        rows = _different_rows(n, 0.9 * entries)
        nbytes = rows * d * size + 1.0 * count * d * size + entries * (12.0 if case["offset"] else 8.0) + 4.0 * count
        if kind == "list":
            return {"bytes": nbytes, "flops": 0.9 * entries * (2.0 * d + 4.0)}
        nbytes += 1.0 * (n + count) * d * size + 8.0 * entries
        return {"bytes": nbytes, "flops": 0.9 * entries * (6.0 * d + 8.0)}
    if kind in ("distill", "distill_train"):
        count, elements = case["count"], 1.0 * case["count"] * case["m"]
        nbytes = elements * (4.0 + BYTES[case["type"]]) + count * (8.0 if case["rest"] else 4.0)
        flops = elements * (10.0 if case["rest"] else 7.0)
        if kind == "distill":
            return {"bytes": nbytes, "flops": flops}
        return {"bytes": nbytes + 4.0 * elements + 4.0 * count, "flops": flops + 3.0 * elements}
    lengths = _token_lengths(case)
    sequences, tokens = len(lengths), 1.0 * sum(lengths)
    read = 5.0 + (4.0 if case["reference"] else 0.0)
    if kind == "preference":
        return {"bytes": tokens * (read + 4.0) + sequences * (4.0 + 4.0) + case["count"] * 12.0, "flops": 3.0 * tokens}
    read += 8.0 if case["each"] else 4.0
    return {"bytes": tokens * (read + 4.0) + sequences * 20.0, "flops": tokens * (18.0 if case["reference"] else 10.0)}


# ---- in 64 bits ----------------------------------------------------------------------------

def _exact_list(case, state):
    n, d, count, m = case["n"], case["d"], case["count"], case["m"]
    f64 = dict(dtype=torch.float64, device="cuda")
    points, queries, ids, scale = state["points"], state["queries"].to(torch.float64), state["ids"], state["scale"]
    train = case["kind"] == "list_train"
    out = {"logp": torch.full((count, m), -math.inf, **f64), "lse": torch.full((count,), -math.inf, **f64)}
    if train:
        out["offset"], out["queries"], out["points"] = torch.zeros((count, m), **f64), torch.zeros((count, d), **f64), torch.zeros((n, d), **f64)
    step = max(1, 100_000_000 // (m * d))
    for at in range(0, count, step):
        line, entry = torch.nonzero(ids[at:at + step] >= 0, as_tuple=True)
        if line.numel() == 0:
            continue
        line = line + at
        row = ids[line, entry].long()
        x = points.index_select(0, row).to(torch.float64)
        q = queries.index_select(0, line)
        s = torch.linalg.vecdot(x, q) * scale
        if state["offset"] is not None:
            s = s + state["offset"][line, entry].to(torch.float64)
        part = torch.full((min(step, count - at), m), -math.inf, **f64)
        part[line - at, entry] = s
        lse = torch.logsumexp(part, 1)
        out["lse"][at:at + step] = lse
        logp = s - lse[line - at]
        out["logp"][line, entry] = logp
        if train:
            g = state["grad_logp"][line, entry].to(torch.float64)
            all_g = torch.zeros(part.shape[0], **f64).index_add_(0, line - at, g)
            g = g - logp.exp() * all_g[line - at]
            out["offset"][line, entry] = g
            g = (g * scale)[:, None]
            out["queries"].index_put_((line,), x * g, accumulate=True)
            out["points"].index_put_((row,), q * g, accumulate=True)
    return out


def _exact_distill(case, state):
    f64 = torch.float64
    z, logp = state["teacher"].to(f64) / case["temperature"], state["logp"].to(f64)
    gone = z.isneginf()
    logp = logp.masked_fill(gone, -math.inf)
    lse = torch.logsumexp(z, 1) if state["teacher_lse"] is None else state["teacher_lse"].to(f64)
    log_t = (z - lse[:, None]).masked_fill(gone, -math.inf)
    t = log_t.exp()
    loss = (t * (log_t - logp)).masked_fill(gone, 0.0).sum(1)
    pull = torch.zeros_like(lse)
    if state["teacher_lse"] is not None:
        rest, left = 1.0 - t.sum(1), 1.0 - logp.exp().sum(1)
        rest = torch.clamp(rest, min=0.0)
        floor = torch.clamp(left, min=LEAST_REST)
        loss = loss + torch.special.xlogy(rest, rest) - rest * floor.log()
        pull = (rest / floor) * (left > LEAST_REST)
    loss = loss.masked_fill(gone.all(1), 0.0)
    if case["kind"] == "distill":
        return loss
    grad = (pull[:, None] * logp.exp() - t).masked_fill(gone, 0.0)
    return {"loss": loss, "grad": grad * state["grad_loss"].to(f64)[:, None]}


def _exact_tokens(case, state):
    f64 = torch.float64
    lengths = (state["offsets"][1:] - state["offsets"][:-1]).long()
    tokens, used = state["logp"].shape[0], int(state["offsets"][-1])
    mask = state["mask"][:used]
    which = torch.repeat_interleave(torch.arange(lengths.shape[0], device="cuda"), lengths)[mask]
    many = torch.bincount(which, minlength=lengths.shape[0]).to(f64)

    def sums(v):
        return torch.bincount(which, weights=v, minlength=lengths.shape[0]).to(f64)

    def spread(v):
        out = torch.zeros(tokens, dtype=f64, device="cuda")
        out[:used][mask] = v
        return out

    logp = state["logp"][:used][mask].to(f64)
    ref = state["ref"][:used][mask].to(f64) if case["reference"] else None
    up = state["grad_loss"].to(f64)
    divide = many.clamp(min=1.0) if case["average"] else torch.ones_like(many)
    if case["kind"] == "preference":
        reward = BETA * sums(logp - ref if case["reference"] else logp) / divide
        x = reward.view(-1, 2)[:, 0] - reward.view(-1, 2)[:, 1] - MARGIN
        log_sigma = torch.nn.functional.logsigmoid
        loss = -(1.0 - SMOOTHING) * log_sigma(x) - SMOOTHING * log_sigma(-x)
        slope = up * BETA * (torch.sigmoid(x) - (1.0 - SMOOTHING))
        return {"loss": loss, "logit": x, "reward": reward, "grad": spread((torch.stack([slope, -slope], 1).view(-1) / divide)[which])}
    a = state["advantage"][:used][mask].to(f64) if case["each"] else state["advantage"].to(f64)[which]
    ratio = (logp - state["old"][:used][mask].to(f64)).exp()
    held = ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH)
    loss = -torch.minimum(ratio * a, held * a)
    over = held * a < ratio * a
    slope = -(ratio * a).masked_fill(over, 0.0)
    kl = torch.zeros_like(loss)
    if case["reference"]:
        kl = torch.expm1(ref - logp) - (ref - logp)
        loss = loss + KL * kl
        slope = slope - KL * torch.expm1(ref - logp)
    return {"loss": sums(loss) / divide, "kl": sums(kl) / divide, "clipped": sums(over.to(f64)) / many.clamp(min=1.0), "grad": spread((up / divide)[which] * slope)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] in ("list", "list_train"):
        return _exact_list(case, state)
    if case["kind"] in ("distill", "distill_train"):
        return _exact_distill(case, state)
    return _exact_tokens(case, state)
