"""Losses of log probabilities against plain forms in 64 bits.

The kernels work in 64 bits with exponentials good to 1e-13 and round once: bounds are half a step of fp32 and 1e-12 of the magnitudes that
a result is the sum of (1e-12 / r of what is divided by r)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF, NAN = math.inf, math.nan
LEAST = 2.0 ** -20


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def within(got, want, bound, what):
    same = (got == want.float()) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, -1.0, (got.double() - want).abs() - bound)
    worst = off.max().item() if off.numel() else 0.0
    assert not math.isnan(worst) and worst <= 0, "%s: over the bound by %g" % (what, worst)


# ---- distillation ------------------------------------------------------------------------------

def distill_inputs(rows, m, kind, tau, seed=0):
    g = gen(rows + 5 * m + seed)
    z = (3.0 * normal((rows, m), g)).to(TYPES[kind])
    s = z.double() / tau + normal((rows, m), g).double()
    other = 0.02 + torch.rand((2, rows), generator=g, device="cuda").double()
    logp = (s - torch.logsumexp(s, 1, keepdim=True) - torch.log1p(other[0])[:, None]).float() if m else torch.zeros((rows, 0), device="cuda")
    lse = (torch.logsumexp(z.double() / tau, 1) + torch.log1p(other[1])).float()
    if m > 1:
        gone = torch.rand((rows, m), generator=g, device="cuda") < 0.2
        gone[:, 0] = False
        if rows > 1:
            gone[1] = True  # nothing of the teacher's
        z[gone] = -INF
        # what the student has there does not count
        logp = torch.where(gone, torch.where(torch.rand((rows, m), generator=g, device="cuda") < 0.5, -INF, NAN), logp)
    return g, logp, z, lse


def distill_want(logp, z, lse, tau, up):
    """(loss, its bound, gradient, its bound)"""
    there = ~(z == -INF)
    zd = z.double() / tau
    lp = torch.where(there, logp.double(), -INF)
    some = there.any(1)
    l = torch.logsumexp(zd, 1) if lse is None else lse.double()
    P = torch.where(there, (zd - l[:, None]).exp(), 0.0)
    term = torch.where(P > 0, P * (zd - l[:, None] - lp), 0.0)
    loss, size = term.sum(1), torch.where(P > 0, P * (zd.abs() + l.abs()[:, None] + lp.abs()), 0.0).sum(1)
    grad, g_size = -P, P.clone()
    if lse is not None:
        p = lp.exp()
        R, left = (1.0 - P.sum(1)).clamp(min=0.0), 1.0 - p.sum(1)
        r = left.clamp(min=LEAST)
        extra = torch.where(R > 0, R * torch.log(R / r), 0.0)
        loss, size = loss + extra, size + extra.abs() + 1.0 + R / r
        pull = torch.where(left > LEAST, R / r, 0.0)[:, None] * p
        grad = torch.where(there, grad + pull, 0.0)
        g_size = g_size + pull * (1.0 + 1.0 / r)[:, None] + p / r[:, None]
    loss = torch.where(some, loss, 0.0)
    up = up.double()[:, None]
    grad = torch.where(there, grad * up, 0.0)
    return loss, U * loss.abs() + 1e-12 * size + 1e-40, grad, U * grad.abs() + 1e-12 * g_size * up.abs() + 1e-40


DISTILL = [(0, 5), (4, 0), (1, 1), (3, 2), (70, 10), (33, 16), (5, 17), (64, 33), (9, 64), (200, 65), (7, 129), (3, 257), (5, 513), (2, 1000), (3, 1025), (2, 4096), (1, 4095), (5000, 3)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,m", DISTILL)
@pytest.mark.parametrize("rest", [False, True])
def test_distill(kind, rows, m, rest):
    for tau in (1.0, 2.5):
        g, logp, z, lse = distill_inputs(rows, m, kind, tau)
        lse = lse if rest else None
        up = normal((rows,), g)
        loss, e_loss, grad, e_grad = distill_want(logp, z, lse, tau, up)
        wide = torch.full((rows, m + 5), NAN, dtype=TYPES[kind], device="cuda")
        wide[:, 3:m + 3] = z
        for view in (z, wide[:, 3:m + 3]):
            got = avq.distill_loss(logp, view, lse, temperature=tau)
            within(got, loss, e_loss, "loss")
            g_got, l_got = avq.distill_loss_grad(logp, view, up, lse, temperature=tau)
            assert torch.equal(got, l_got)
            within(g_got, grad, e_grad, "gradient")


@pytest.mark.parametrize("rows,m", [(65_536 * 64 + 77, 5), (70_001, 1100)])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_of_more_rows_than_workgroups(rows, m, rest):
    g, logp, z, lse = distill_inputs(rows, m, "bf16", 1.0)
    lse = lse if rest else None
    up = normal((rows,), g)
    got, l_got = avq.distill_loss_grad(logp, z, up, lse)
    for at in (0, rows // 2, rows - 3000):  # (parts, for the memory of the 64-bit form)
        part = slice(at, at + 3000)
        loss, e_loss, grad, e_grad = distill_want(logp[part], z[part], None if lse is None else lse[part], 1.0, up[part])
        within(l_got[part], loss, e_loss, "loss")
        within(got[part], grad, e_grad, "gradient")


def test_distill_where_student_and_teacher_agree():
    """The loss is what is left of terms a million times as large."""
    g = gen(1)
    z = 2.0 * normal((50, 40), g)
    base = torch.log_softmax(z.double(), 1)
    logp = (base + 1e-4 * normal((50, 40), g).double()).float()
    up = torch.ones(50, device="cuda")
    loss, e_loss, grad, e_grad = distill_want(logp, z, None, 1.0, up)
    assert loss.abs().max() < 1e-3
    got, l_got = avq.distill_loss_grad(logp, z, up)
    within(l_got, loss, e_loss, "loss")
    within(got, grad, e_grad, "gradient")


def test_distill_where_a_list_has_all_of_the_probability():
    """r is at its floor for rows whose list is the whole table, and the gradient is that of the terms of the list alone."""
    g = gen(2)
    z = normal((6, 30), g)
    logp = torch.log_softmax(normal((6, 30), g).double(), 1).float()
    lse = torch.logsumexp(z.double(), 1).float()
    up = torch.ones(6, device="cuda")
    loss, e_loss, grad, e_grad = distill_want(logp, z, lse, 1.0, up)
    got, l_got = avq.distill_loss_grad(logp, z, up, lse)
    within(l_got, loss, e_loss, "loss")
    within(got, grad, e_grad, "gradient")
    assert torch.allclose(-got, torch.softmax(z, 1), rtol=0, atol=1e-6)


def test_distill_of_infinities_and_nan():
    z = torch.tensor([[0.0, 1.0], [0.0, 1.0], [NAN, 1.0], [NAN, NAN], [0.0, -3e38], [0.0, 1.0]], device="cuda")
    logp = torch.tensor([[-1.0, -INF], [-1.0, NAN], [-1.0, -1.0], [-1.0, -1.0], [-1.0, -INF], [-1.0, -0.5]], device="cuda")
    up = torch.ones(6, device="cuda")
    grad, loss = avq.distill_loss_grad(logp, z, up)
    assert loss[0] == INF and bool(torch.isnan(loss[1:4]).all())
    assert bool(torch.isfinite(grad[0]).all())                     # a row of probability 0 is pulled up all the same
    assert bool(torch.isnan(grad[2:4]).all())
    assert loss[4] == 1.0 and grad[4, 1] == 0                      # a teacher's mask of the type's lowest value
    assert bool(torch.isfinite(loss[5]))


def test_distill_gradient_against_differences():
    for rest in (False, True):
        g, logp, z, lse = distill_inputs(4, 9, "f32", 1.5, 3)
        lse = lse if rest else None
        up = normal((4,), g)
        got = avq.distill_loss_grad(logp, z, up, lse, temperature=1.5)[0]
        there = ~(z == -INF)
        for i in torch.nonzero(there.reshape(-1))[:, 0].tolist():
            h, sides = 1e-5, []
            for sign in (1, -1):
                moved = logp.double().clone()
                moved.view(-1)[i] += sign * h
                sides.append((distill_want(moved, z, lse, 1.5, up)[0] * up.double()).sum().item())
            slope = (sides[0] - sides[1]) / (2 * h)
            # third derivatives of R log(R / r) are below 2 / r^3 with r above 0.01
            assert abs(got.view(-1)[i].item() - slope) < 1e-3 * h * h * 2e9 + 1e-7 * (1 + abs(slope)), (rest, i)


# ---- sequences -----------------------------------------------------------------------------------

# lengths of the sequences; an even number of them
LENGTHS = {
    "none": [], "empty": [0, 0], "one": [1, 1], "few": [3, 0, 1, 7], "ragged": [64, 1, 255, 256, 257, 0, 1000, 5], "long": [70_000, 3, 2, 9000],
    "many": [(i * 7) % 13 for i in range(3000)], "tiles": [2048, 2048, 4096, 1, 2047, 4097], "huge": [300_001, 1],
}


def sequences(name, seed=0, before=3, behind=5):
    g = gen(len(LENGTHS[name]) + seed)
    lengths = torch.tensor(LENGTHS[name], dtype=torch.int64, device="cuda")
    offsets = torch.zeros(lengths.numel() + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = lengths.cumsum(0)
    offsets += before
    tokens = before + int(lengths.sum()) + behind
    which = torch.full((tokens,), -1, dtype=torch.int64, device="cuda")
    if lengths.numel():
        which[before:tokens - behind] = torch.repeat_interleave(torch.arange(lengths.numel(), device="cuda"), lengths)
    mask = torch.rand(tokens, generator=g, device="cuda") < 0.8
    if "ragged" in name:
        mask[offsets[2]:offsets[3]] = False  # a sequence of which nothing counts
    return g, offsets, which, mask, tokens


def masked(t, mask, which, junk):
    return torch.where(mask & (which >= 0), t, junk)


def total(v, counted, which, count):
    return torch.zeros(max(count, 1), dtype=torch.float64, device="cuda").index_add_(0, which.clamp(min=0), torch.where(counted, v, 0.0))[:count]


def preference_want(logp, offsets, which, ref, mask, beta, margin, smoothing, average, up):
    count = offsets.shape[0] - 1
    counted = (which >= 0) if mask is None else (which >= 0) & mask
    v = logp.double() - (ref.double() if ref is not None else 0.0)
    many = total(torch.ones_like(v), counted, which, count).clamp(min=1.0) if average else torch.ones(count, dtype=torch.float64, device="cuda")
    reward = beta * total(v, counted, which, count) / many
    size = abs(beta) * total(torch.where(counted, v.abs(), 0.0), counted, which, count) / many
    x = reward[0::2] - reward[1::2] - margin
    sp = torch.nn.functional.softplus
    loss = (1 - smoothing) * sp(-x) + smoothing * sp(x)
    slope = beta * (smoothing * torch.sigmoid(x) - (1 - smoothing) * torch.sigmoid(-x)) * up.double()
    each = torch.stack([slope, -slope], 1).reshape(-1) / many
    e = 1e-12 * (size[0::2] + size[1::2] + abs(margin) + 1)
    grad = torch.where(counted, each[which.clamp(min=0)], 0.0) if count else torch.zeros_like(v)
    e_each = torch.stack([e, e], 1).reshape(-1) * abs(beta) * up.double().abs().repeat_interleave(2) / many
    e_grad = U * grad.abs() + (torch.where(counted, e_each[which.clamp(min=0)], 0.0) if count else 0.0) + 1e-40
    return loss, U * loss.abs() + e, x, U * x.abs() + e, reward, U * reward.abs() + 1e-12 * size, grad, e_grad


@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("with_ref,with_mask,average,smoothing", [(True, True, False, 0.1), (False, False, True, 0.0), (True, False, True, 1.0), (False, True, False, 0.5)])
def test_preference(name, with_ref, with_mask, average, smoothing):
    g, offsets, which, mask, tokens = sequences(name)
    # (masked tokens hold what log_probs gives for padding, and NaN)
    junk = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.5, -INF, NAN)
    there = which >= 0 if not with_mask else mask & (which >= 0)
    logp = torch.where(there, -2.0 * normal((tokens,), g).abs(), junk)
    ref = torch.where(there, logp + 0.1 * normal((tokens,), g), junk) if with_ref else None
    mask = mask if with_mask else None
    up = normal(((offsets.shape[0] - 1) // 2,), g)
    args = dict(ref=ref, mask=mask, beta=0.3, margin=0.2, smoothing=smoothing, average=average)
    loss, e_loss, x, e_x, reward, e_reward, grad, e_grad = preference_want(logp, offsets, which, ref, mask, 0.3, 0.2, smoothing, average, up)
    r = avq.preference_loss(logp, offsets, **args)
    got, r2 = avq.preference_loss_grad(logp, offsets, up, **args)
    assert all(torch.equal(a, b) for a, b in zip(r, r2)), "loss alone and with the gradient differ"
    within(r.loss, loss, e_loss, "loss")
    within(r.logit, x, e_x, "logit")
    within(r.reward, reward, e_reward, "reward")
    within(got, grad, e_grad, "gradient")


def test_preference_far_apart():
    """Logits of thousands either way: loss and gradient stay what they are, and infinities do not become NaN."""
    logp = torch.tensor([-1.0, -90_000.0, -90_000.0, -1.0, -INF, -1.0, -1.0, -INF], device="cuda")
    offsets = torch.arange(9, dtype=torch.int32, device="cuda")
    up = torch.ones(4, device="cuda")
    grad, r = avq.preference_loss_grad(logp, offsets, up, beta=0.1)
    assert r.loss[0] == 0 and grad[0] == 0
    assert abs(r.loss[1].item() - 0.1 * 89_999.0) < 1e-3 and abs(grad[2].item() + 0.1) < 1e-8 and abs(grad[3].item() - 0.1) < 1e-8
    assert r.loss[2] == INF and r.logit[2] == -INF and r.loss[3] == 0 and r.logit[3] == INF
    assert bool(torch.isfinite(grad).all())


def policy_want(logp, old, advantage, offsets, which, ref, mask, low, high, kl_weight, average, up):
    count = offsets.shape[0] - 1
    counted = (which >= 0) if mask is None else (which >= 0) & mask
    at = which.clamp(min=0)
    lp, o = torch.where(counted, logp, 0.0).double(), torch.where(counted, old, 0.0).double()
    a = advantage.double() if advantage.shape[0] == logp.shape[0] else (advantage.double()[at] if count else torch.zeros_like(lp))
    a = torch.where(counted, a, 0.0)
    r = (lp - o).exp()
    over = ((a > 0) & (r > 1 + high)) | ((a < 0) & (r < 1 - low))
    loss = -torch.minimum(r * a, r.clamp(1 - low, 1 + high) * a)
    slope = torch.where(over, 0.0, -r * a)
    kl = torch.zeros_like(loss)
    if ref is not None:
        away = torch.where(counted, ref, 0.0).double() - lp
        kl = torch.expm1(away) - away
        loss = loss + kl_weight * kl
        slope = slope - kl_weight * torch.expm1(away)
    many = total(torch.ones_like(lp), counted, which, count).clamp(min=1.0)
    share = 1.0 / many if average else torch.ones_like(many)
    size = total((r * a).abs() + kl.abs() + 1e-6, counted, which, count) * share
    each = up.double() * share
    grad = torch.where(counted, slope * each[at], 0.0) if count else torch.zeros_like(lp)
    e_grad = U * grad.abs() + (1e-12 * ((r * a).abs() + 1.0 + kl.abs()) * each[at].abs() if count else 0.0) + 1e-40
    L, K = total(loss, counted, which, count) * share, total(kl, counted, which, count) * share
    C = total(over.double(), counted, which, count) / many
    return L, U * L.abs() + 1e-12 * size, K, U * K.abs() + 1e-12 * size, C, U * C, grad, e_grad


@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("with_ref,with_mask,each,average", [(True, True, True, True), (False, False, False, False), (True, False, False, True), (True, True, True, False)])
def test_policy(name, with_ref, with_mask, each, average):
    g, offsets, which, mask, tokens = sequences(name, 1)
    there = which >= 0 if not with_mask else mask & (which >= 0)
    junk = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.5, -INF, NAN)
    logp = torch.where(there, -2.0 * normal((tokens,), g).abs(), junk)
    old = torch.where(there, logp + 0.3 * normal((tokens,), g), junk)
    ref = torch.where(there, logp + 0.1 * normal((tokens,), g), junk) if with_ref else None
    count = offsets.shape[0] - 1
    advantage = normal((tokens if each else count,), g)
    if each:
        advantage = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.1, 0.0, advantage)
        advantage = torch.where(there, advantage, NAN)
    mask = mask if with_mask else None
    kl = 0.07 if with_ref else 0.0
    up = normal((count,), g)
    args = dict(ref=ref, mask=mask, clip=(0.2, 0.3), kl=kl, average=average, each=each)
    L, e_L, K, e_K, C, e_C, grad, e_grad = policy_want(logp, old, advantage, offsets, which, ref, mask, 0.2, 0.3, kl, average, up)
    r = avq.policy_loss(logp, old, advantage, offsets, **args)
    got, r2 = avq.policy_loss_grad(logp, old, advantage, offsets, up, **args)
    assert all(torch.equal(a, b) for a, b in zip(r, r2)), "loss alone and with the gradient differ"
    within(r.loss, L, e_L, "loss")
    within(r.kl, K, e_K, "kl")
    within(r.clipped, C, e_C, "clipped")
    within(got, grad, e_grad, "gradient")


def test_policy_far_apart():
    """Ratios and divergences that are infinite count for nothing where they have no weight."""
    logp = torch.tensor([-1.0, -1.0, -1.0, -2000.0, -INF, NAN], device="cuda")
    old = torch.tensor([-2000.0, -2000.0, -2000.0, -1.0, -1.0, -1.0], device="cuda")
    ref = torch.tensor([-1.0, -INF, -1.0, -1.0, -1.0, -1.0], device="cuda")
    advantage = torch.tensor([0.0, 1.0, -1.0, 1.0, 1.0, 0.0], device="cuda")
    offsets = torch.arange(7, dtype=torch.int32, device="cuda")
    up = torch.ones(6, device="cuda")
    grad, r = avq.policy_loss_grad(logp, old, advantage, offsets, up, ref=ref, clip=0.25)
    assert r.loss[0] == 0 and grad[0] == 0                            # no advantage
    assert r.loss[1] == -1.25 and grad[1] == 0 and r.kl[1] == INF     # clipped; the divergence has no weight here
    assert r.loss[2] == INF and grad[2] == INF                        # a bad answer that has become certain
    assert r.loss[3] == 0 and grad[3] == 0 and r.loss[4] == 0 and grad[4] == 0
    assert bool(torch.isnan(r.loss[5])) and bool(torch.isnan(grad[5]))
    assert r.clipped.tolist() == [0.0, 1.0, 0.0, 0.0, 0.0, 0.0]


def test_token_gradients_against_differences():
    g, offsets, which, _, tokens = sequences("few", 2)
    logp = -normal((tokens,), g).abs()
    old, ref = logp + 0.05 * normal((tokens,), g), logp + 0.2 * normal((tokens,), g)
    advantage = normal((tokens,), g)
    up2, up4 = normal((2,), g), normal((4,), g)
    a = avq.preference_loss_grad(logp, offsets, up2, ref=ref, beta=0.5, smoothing=0.2, average=True)[0]
    b = avq.policy_loss_grad(logp, old, advantage, offsets, up4, ref=ref, clip=0.4, kl=0.3)[0]
    h = 1e-6
    for i in range(tokens):
        slopes = []
        for sign in (1, -1):
            moved = logp.double()
            moved[i] += sign * h
            slopes.append((
                (preference_want(moved, offsets, which, ref, None, 0.5, 0.0, 0.2, True, up2)[0] * up2.double()).sum().item(),
                (policy_want(moved, old, advantage, offsets, which, ref, None, 0.4, 0.4, 0.3, True, up4)[0] * up4.double()).sum().item()))
        # the difference is off by its own rounding, 1e-15 / h, and h^2 of third derivatives of order 1
        assert abs(a[i].item() - (slopes[0][0] - slopes[1][0]) / (2 * h)) < 1e-7
        assert abs(b[i].item() - (slopes[0][1] - slopes[1][1]) / (2 * h)) < 1e-6


def test_offsets_that_leave_the_tokens_are_held_to_them():
    logp = -torch.arange(1.0, 11.0, device="cuda")
    offsets = torch.tensor([-5, 4, 1 << 30], dtype=torch.int32, device="cuda")
    grad, r = avq.preference_loss_grad(logp, offsets, torch.ones(1, device="cuda"), beta=1.0)
    assert r.reward.tolist() == [-10.0, -45.0]
    assert bool((grad[:4] == grad[0]).all()) and bool((grad[4:] == -grad[0]).all())
    p = avq.policy_loss(logp, logp, torch.ones(2, device="cuda"), offsets)
    assert p.loss.tolist() == [-1.0, -1.0]


@pytest.mark.parametrize("name", ["tiles", "long", "few"])
def test_captured_losses_follow_their_inputs(name):
    g, offsets, which, mask, tokens = sequences(name, 3)
    count = offsets.shape[0] - 1
    logp, old = -normal((tokens,), g).abs(), -normal((tokens,), g).abs()
    advantage, up3, up6 = normal((tokens,), g), normal((count // 2,), g), normal((count,), g)
    z, student, up8 = normal((8, 77), g), torch.log_softmax(normal((8, 77), g), 1), normal((8,), g)

    def calls():
        a = avq.preference_loss_grad(logp, offsets, up3, ref=old, mask=mask)
        b = avq.policy_loss_grad(logp, old, advantage, offsets, up6, ref=old, mask=mask, kl=0.1)
        c = avq.distill_loss_grad(student, z, up8)
        return [a[0], *a[1], b[0], *b[1], *c]

    calls()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        calls()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            held = calls()
    torch.cuda.synchronize()
    for step in range(4):
        logp.copy_(-normal((tokens,), g).abs())
        student.copy_(torch.log_softmax(normal((8, 77), g), 1))
        want = calls()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


@pytest.mark.parametrize("name", ["ragged", "long"])
def test_on_another_stream(name):
    g, offsets, which, mask, tokens = sequences(name, 4)
    count = offsets.shape[0] - 1
    logp, old = -normal((tokens,), g).abs(), -normal((tokens,), g).abs()
    z, student = normal((9, 70), g), torch.log_softmax(normal((9, 70), g), 1)
    ups = [normal((n,), g) for n in (count // 2, count, 9)]

    def calls(**how):
        a = avq.preference_loss_grad(logp, offsets, ups[0], ref=old, mask=mask, **how)
        b = avq.policy_loss_grad(logp, old, ups[1], offsets, ups[1], ref=old, mask=mask, kl=0.1, **how)
        return [a[0], *a[1], b[0], *b[1], *avq.distill_loss_grad(student, z, ups[2], **how)]

    want = calls()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = calls(stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_tokens_behind_the_last_sequence_are_zeros_however_many():
    offsets = torch.tensor([70_000, 70_003, 70_005], dtype=torch.int32, device="cuda")
    logp = -torch.ones(3_000_000, device="cuda")
    up = torch.ones(1, device="cuda")
    grad, r = avq.preference_loss_grad(logp, offsets, up, beta=1.0)
    assert r.reward.tolist() == [-3.0, -2.0]
    assert int((grad != 0).sum()) == 5 and bool((grad[70_000:70_005] != 0).all())
    grad = avq.policy_loss_grad(logp, logp, torch.ones(2, device="cuda"), offsets, torch.ones(2, device="cuda"))[0]
    assert int((grad != 0).sum()) == 5 and bool((grad[70_000:70_005] != 0).all())


# ---- more rounds of a workgroup's tokens than one ----------------------------------------------------

# A workgroup of 64, 256 or 1,024 threads takes four tokens a thread at a time: sequences that take it several rounds, and parts that do
ROUNDS = {
    "waves": [5] * 298 + [257, 700],                                                  # 64 threads, rounds of 256
    "fours": [150] * 532 + [1024, 1025, 5000, 2049],                                  # 256 threads, rounds of 1,024
    "groups": [600] * 516 + [4096, 4097, 8193, 10_000],                               # 1,024 threads, rounds of 4,096
    "parts": [50] * 198 + [100_000, 7],                                               # parts of up to 20,000 tokens
}


def threads_of(name, pairs):
    """Threads of a workgroup by the lengths alone, or None for parts."""
    tokens, many = sum(ROUNDS[name]) + 8, len(ROUNDS[name]) // (2 if pairs else 1)
    if many < 256 and tokens > (24_576 if pairs else 8192):
        return None
    mean = tokens / (4 * many if pairs else many)
    return 64 if mean <= 64 else 256 if mean <= 256 else 1024


def test_the_rounds_are_of_every_kind():
    assert [threads_of(name, False) for name in ROUNDS] == [64, 256, 1024, None]
    assert [threads_of(name, True) for name in ROUNDS] == [64, 256, 1024, None]


@pytest.mark.parametrize("name", ROUNDS)
@pytest.mark.parametrize("with_ref,with_mask,each,average", [(True, True, True, True), (False, False, False, False), (True, False, False, True)])
def test_policy_of_several_rounds(name, with_ref, with_mask, each, average, monkeypatch):
    monkeypatch.setitem(LENGTHS, name, ROUNDS[name])
    test_policy(name, with_ref, with_mask, each, average)


@pytest.mark.parametrize("name", ROUNDS)
@pytest.mark.parametrize("with_ref,with_mask,average,smoothing", [(True, True, False, 0.1), (False, False, True, 0.0)])
def test_preference_of_several_rounds(name, with_ref, with_mask, average, smoothing, monkeypatch):
    monkeypatch.setitem(LENGTHS, name, ROUNDS[name])
    test_preference(name, with_ref, with_mask, average, smoothing)
