"""The small model's losses, end to end: each of its gradients against torch's autograd in 64 bits over the whole model."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")

WORDS, DIM = 300, 24


def model_and_inputs(seed, count=64):
    from paper_1908_10396_amd import learn
    model = learn.Model(WORDS, DIM, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    with torch.no_grad():
        model.weight.add_(0.2 * torch.randn(DIM, generator=g, device="cuda"))
        model.bias.add_(0.2 * torch.randn(DIM, generator=g, device="cuda"))
    words = lambda *shape: torch.randint(0, WORDS, shape, generator=g, device="cuda", dtype=torch.int32)
    return model, g, words


def logits(model, a):
    """All logits in 64 bits, from parameters that torch differentiates."""
    leaves = [p.detach().double().requires_grad_() for p in (model.table, model.weight, model.bias)]
    x = leaves[0][a.long()]
    mean = x.mean(1, keepdim=True)
    xhat = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    q = xhat * leaves[1] + leaves[2]
    return leaves, (q @ leaves[0].t()) * model.scale


def agree(got, loss, leaves):
    """fp32 against 64 bits: sums of up to 300 rows and 64 queries whose terms are below 1, by pairs of f16 at 2^-21: 1e-5 of the largest
    entry, and of the loss."""
    loss.backward()
    assert abs(got[0].item() - loss.item()) < 1e-5 * (1 + abs(loss.item()))
    for g, leaf in zip(got[1:], leaves):
        assert g.shape == leaf.shape
        assert float((g.double() - leaf.grad).abs().max()) < 1e-5 * float(leaf.grad.abs().max()) + 1e-7


def test_sampled():
    model, g, words = model_and_inputs(1)
    a, b, drawn = words(64), words(64), words(64, 20)
    drawn[3, 5], drawn[9, 0] = b[3], b[9]
    leaves, s = logits(model, a)
    ids = torch.cat([b[:, None], drawn], 1).long()
    mine = s.gather(1, ids)
    mine = torch.cat([mine[:, :1], mine[:, 1:].masked_fill(drawn == b[:, None], -math.inf)], 1)
    agree(model.sampled_gradients(a, b, drawn), -torch.log_softmax(mine, 1)[:, 0].mean(), leaves)


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("rest", [False, True])
def test_distilled_from_what_an_index_returned(listed, rest):
    if listed and rest:
        rest = False  # (a list has all of the student's probability: nothing is left for other rows)
    from paper_1908_10396_amd import learn
    model, g, words = model_and_inputs(2)
    teacher = learn.Model(WORDS, 32, seed=5)
    idx = learn.index_of(teacher, 16)
    try:
        a, tau = words(64), 1.5
        ids, logp, _ = learn.answer(teacher, idx, a, 10, 64)
    finally:
        idx.close()
    z = (logp * 1.5).to(torch.bfloat16)
    lse = (torch.logsumexp(z.double() / tau, 1) + 0.3).float() if rest else None
    leaves, s = logits(model, a)
    s = s / tau
    mine = torch.log_softmax(s.gather(1, ids.long()), 1) if listed else torch.log_softmax(s, 1).gather(1, ids.long())
    log_t = z.double() / tau - (torch.logsumexp(z.double() / tau, 1) if lse is None else lse.double())[:, None]
    loss = (log_t.exp() * (log_t - mine)).sum(1)
    if rest:
        R, r = 1 - log_t.exp().sum(1), 1 - mine.exp().sum(1)
        loss = loss + R * torch.log(R / r)
    agree(model.distill_gradients(a, ids, z, lse, temperature=tau, listed=listed), loss.mean(), leaves)


def sequences(words):
    a, b = words(64), words(64)
    b[5], b[40] = -1, WORDS + 3  # padding
    offsets = torch.tensor([2, 9, 9, 20, 21, 50, 60], dtype=torch.int32, device="cuda")
    spans = [(2, 9), (9, 9), (9, 20), (20, 21), (21, 50), (50, 60)]
    return a, b, offsets, spans


def test_preferences():
    model, g, words = model_and_inputs(3)
    a, b, offsets, spans = sequences(words)
    ref = model.log_probs(a, b) + 0.1 * torch.randn(64, generator=g, device="cuda")
    leaves, s = logits(model, a)
    real = (b >= 0) & (b < WORDS)
    lp = torch.log_softmax(s, 1).gather(1, torch.where(real, b, 0).long()[:, None])[:, 0]
    ratio = torch.where(real, lp - torch.where(real, ref, 0.0).double(), 0.0)
    sums = torch.stack([ratio[lo:hi].sum() for lo, hi in spans])
    x = 0.5 * (sums[0::2] - sums[1::2])
    loss = (-(0.9 * torch.nn.functional.logsigmoid(x) + 0.1 * torch.nn.functional.logsigmoid(-x))).mean()
    agree(model.preference_gradients(a, b, offsets, ref=ref, beta=0.5, smoothing=0.1), loss, leaves)


def test_policy():
    model, g, words = model_and_inputs(4)
    a, b, offsets, spans = sequences(words)
    now = model.log_probs(a, b)
    old, ref = now + 0.2 * torch.randn(64, generator=g, device="cuda"), now + 0.1 * torch.randn(64, generator=g, device="cuda")
    advantage = torch.randn(6, generator=g, device="cuda")
    leaves, s = logits(model, a)
    real = (b >= 0) & (b < WORDS)
    lp = torch.log_softmax(s, 1).gather(1, torch.where(real, b, 0).long()[:, None])[:, 0]
    r = torch.exp(torch.where(real, lp - torch.where(real, old, 0.0).double(), 0.0))
    away = torch.where(real, torch.where(real, ref, 0.0).double() - lp, 0.0)
    losses = []
    for (lo, hi), A in zip(spans, advantage.double()):
        l = -torch.minimum(r[lo:hi] * A, r[lo:hi].clamp(0.8, 1.3) * A) + 0.05 * (torch.expm1(away[lo:hi]) - away[lo:hi])
        l = l[real[lo:hi]]
        losses.append(l.mean() if l.numel() else l.sum())
    agree(model.policy_gradients(a, b, old, advantage, offsets, ref=ref, clip=(0.2, 0.3), kl=0.05), torch.stack(losses).mean(), leaves)


def test_a_student_and_walks():
    from paper_1908_10396_amd import learn
    corpus = learn.Corpus(400, topic=8, seed=1)
    model = learn.Model(400, 16, seed=1)
    for _ in range(3):
        model.step(*corpus.pairs(256))
    idx = learn.index_of(model, 8)
    try:
        student = learn.Model(400, 8, seed=2)
        losses = [learn.taught(student, model, idx, corpus.pairs(128)[0], k=8, reorder_k=64) for _ in range(2)]
        assert all(math.isfinite(float(x)) for x in losses)
        before, words = learn.walks(model, idx, corpus.pairs(10)[0], 5, corpus.gen, k=8, reorder_k=64)
        assert before.shape == words.shape == (10, 5) and bool((before[:, 1:] == words[:, :-1]).all())
        assert bool((words >= 0).all()) and bool((words < 400).all())
    finally:
        idx.close()
    for how in ("preference", "policy"):
        shares = learn.tune(model, corpus, how, rounds=2, count=16, length=3)
        assert len(shares) == 2 and all(0.0 <= x <= 1.0 for x in shares)
        assert all(bool(torch.isfinite(p).all()) for p in (model.table, model.weight, model.bias))


def tuning(seed):
    """A model away from its reference's parameters, walks of three words and their rewards, of which some are equal."""
    model, g, words = model_and_inputs(seed)
    first = [p.detach().clone() for p in (model.table, model.weight, model.bias)]
    with torch.no_grad():
        for p in (model.table, model.weight, model.bias):
            p.add_(0.1 * torch.randn(p.shape, generator=g, device="cuda"))
    reward = torch.tensor([[0.0, 1.0], [2 / 3, 1 / 3], [1 / 3, 1 / 3], [1.0, 2 / 3], [0.0, 0.0], [1 / 3, 1.0]], device="cuda")
    return model, first, words(12, 3), words(12, 3), reward


def walks_log_probs(model, first, before, after):
    """Leaves, log p of the walks' words in 64 bits from the model's parameters, and from the reference's: [12][3]."""
    leaves, s = logits(model, before.view(-1))
    at = after.view(-1, 1).long()
    now = torch.log_softmax(s, 1).gather(1, at).view(12, 3)
    held = [p.data for p in (model.table, model.weight, model.bias)]
    for p, value in zip((model.table, model.weight, model.bias), first):
        p.data = value
    ref = torch.log_softmax(logits(model, before.view(-1))[1], 1).gather(1, at).view(12, 3).detach()
    for p, value in zip((model.table, model.weight, model.bias), held):
        p.data = value
    return leaves, now, ref


@pytest.mark.parametrize("how", ["preference", "policy"])
def test_tuning_steps_have_the_gradient_of_their_definition(how, monkeypatch):
    """Which walk is preferred or rewarded, that pairs of equal rewards are left out, whose log probabilities the reference's are, and
    that the step is taken from the model's own parameters."""
    from paper_1908_10396_amd import learn
    model, first, before, after, reward = tuning(6)
    held = [p.detach().clone() for p in (model.table, model.weight, model.bias)]
    applied = []
    monkeypatch.setattr(model, "apply", lambda *got: applied.append(got))
    learn.tune_on(model, how, before, after, reward, first, steps=1)
    assert all(torch.equal(p, h) for p, h in zip((model.table, model.weight, model.bias), held))
    leaves, now, ref = walks_log_probs(model, first, before, after)
    losses = []
    for pair in range(6):
        a, b = 2 * pair, 2 * pair + 1
        if how == "preference":
            if reward[pair, 0] == reward[pair, 1]:
                continue
            w, l = (a, b) if reward[pair, 0] > reward[pair, 1] else (b, a)
            x = 0.5 * ((now[w] - ref[w]).sum() - (now[l] - ref[l]).sum())
            losses.append(-0.9 * torch.nn.functional.logsigmoid(x) - 0.1 * torch.nn.functional.logsigmoid(-x))
        else:
            for walk, other in ((a, b), (b, a)):
                A = (reward[pair, walk - a] - reward[pair, other - a]).double() / 2
                r = torch.exp(now[walk] - now[walk].detach())
                away = ref[walk] - now[walk]
                losses.append((-r * A + 0.04 * (torch.expm1(away) - away)).mean())
    assert len(applied) == 1
    agree(applied[0], torch.stack(losses).mean(), leaves)


def test_walks_of_equal_rewards_are_not_compared(monkeypatch):
    from paper_1908_10396_amd import learn
    model, first, before, after, reward = tuning(7)
    monkeypatch.setattr(model, "apply", lambda *got: pytest.fail("a step on walks that are equal"))
    learn.tune_on(model, "preference", before, after, torch.full_like(reward, 0.5), first)
