"""Log probabilities over lists of rows, and their gradient, against plain forms in 64 bits.

Tolerances are bounds, element by element (u = 2^-24): a sum of m terms in any order is off by at most m u times the sum of
their magnitudes, a result by half a step of its type; expf, expm1f and log1pf by two steps."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-38, "bf16": 1e-38, "f16": 2.0 ** -24}
INF = math.inf

# (n, d, queries, list)
SHAPES = [
    (1, 1, 1, 1), (5, 3, 2, 0), (5, 3, 0, 4), (10, 100, 3, 7), (1000, 101, 17, 130), (300, 32, 65, 64), (777, 1024, 9, 33), (50, 1030, 5, 257), (20, 16384, 2, 9),
    (40_000, 64, 1, 4096), (5000, 16, 700, 5), (100, 475, 40, 100), (3, 7, 33, 1), (70_000, 8, 2, 2049), (900, 256, 3, 1000), (4000, 512, 300, 20),
    (3000, 33, 4100, 7), (500, 130, 5000, 64), (70, 1100, 4097, 3), (200, 100, 100, 90), (50_000, 260, 40, 300), (30, 2050, 60, 50),
]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def lists(shape, n, g, padding=0.2):
    ids = torch.randint(0, n, shape, generator=g, device="cuda", dtype=torch.int32)
    draw = torch.rand(shape, generator=g, device="cuda")
    ids = torch.where(draw < padding / 2, -1, ids)
    ids = torch.where((draw >= padding / 2) & (draw < padding), n + 5, ids)
    if shape[0] > 2:
        ids[1] = -7  # a list of padding alone
    return ids


def within(got, want, bound, what):
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))  # (infinities)
    off = torch.where(same, -1.0, (got.double() - want).abs() - bound)
    worst = off.max().item() if off.numel() else 0.0
    assert not math.isnan(worst) and worst <= 0, "%s: over the bound by %g" % (what, worst)


def strided(t, extra, shift=0):
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, shift:shift + t.shape[1]] = t
    return wide[:, shift:shift + t.shape[1]]


def inputs(n, d, nq, m, kind, seed=0):
    g = gen(n + 3 * d + 7 * nq + 11 * m + seed)
    return g, normal((n, d), g, TYPES[kind]), normal((nq, d), g, TYPES[kind]), lists((nq, m), n, g), 2.0 / math.sqrt(d)


def scores(x, q, ids, scale, offset):
    """(scores in 64 bits, -inf for padding; how far fp32 may be from them; which entries are rows)"""
    nq, m = ids.shape
    s32 = torch.tensor(scale, dtype=torch.float32).item()
    real = (ids >= 0) & (ids < x.shape[0])
    rows = x.double()[torch.where(real, ids, 0).long()]
    s = torch.bmm(rows, q.double()[:, :, None])[:, :, 0] * s32
    e = (x.shape[1] + 8) * U * torch.bmm(rows.abs(), q.double().abs()[:, :, None])[:, :, 0] * abs(s32)
    if offset is not None:
        s = s + offset.double()
    e = e + 2 * U * torch.where(s.abs() < INF, s.abs(), 0.0)
    return torch.where(real, s, -INF), torch.where(real & (s > -INF), e, 0.0), real


def check_probs(r, x, q, ids, scale, offset=None):
    s, e, real = scores(x, q, ids, scale, offset)
    nq, m = ids.shape
    assert r.logp.shape == (nq, m) and r.lse.shape == (nq,)
    if m == 0:
        assert bool((r.lse == -INF).all())
        return
    lse = torch.logsumexp(s, 1)
    some = lse > -INF
    logp = torch.where(some[:, None], s - lse[:, None], -INF)
    most, size = e.amax(1), torch.where(s > -INF, s.abs(), 0.0).amax(1)
    e_sum = most + (m + 16) * U
    within(r.lse, lse, e_sum + 4 * U * size, "lse")
    finite = torch.where(logp > -INF, logp.abs(), 0.0)
    within(r.logp, logp, e + e_sum[:, None] + 4 * U * size[:, None] + 4 * U * finite, "logp")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,nq,m", SHAPES)
def test_list_log_probs(kind, n, d, nq, m):
    g, x, q, ids, scale = inputs(n, d, nq, m, kind)
    check_probs(avq.list_log_probs(x, q, ids, scale=scale), x, q, ids, scale)
    offset = 3.0 * normal((nq, m), g)
    r = avq.list_log_probs(strided(x, 5, 3), strided(q, 7, 1), ids, offset=offset, scale=-scale)
    check_probs(r, x, q, ids, -scale, offset)
    again = avq.list_log_probs(strided(x, 5, 3), strided(q, 7, 1), ids, offset=offset, scale=-scale)
    assert torch.equal(r.logp, again.logp) and torch.equal(r.lse, again.lse), "two calls differ"


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq,m,d", [(3, 50, 40), (200, 33, 40), (1, 3000, 40), (5000, 12, 40), (1100, 1500, 40), (6, 20, 4100)])
def test_masks_infinities_and_nan(kind, nq, m, d):
    g, x, q, ids, scale = inputs(500, d, nq, m, kind)
    offset = normal((nq, m), g)
    offset[:, ::3] = -INF
    offset[:, 1::7] = torch.finfo(torch.float32).min
    if nq > 2:
        offset[2] = -INF  # nothing is left of a list of rows
        ids[2] = ids[2].clamp(0, 499)
    r = avq.list_log_probs(x, q, ids, offset=offset, scale=scale)
    check_probs(r, x, q, ids, scale, offset)
    # what lies in padding and in masks does not matter, NaN of a row that no list names neither
    bad = offset.clone()
    bad[(ids < 0) | (ids >= 500)] = float("nan")
    x2 = torch.cat([x, x[:1]])
    x2[500] = float("nan")
    r2 = avq.list_log_probs(x2[:500], q, ids, offset=bad, scale=scale)
    assert torch.equal(r.logp, r2.logp) and torch.equal(r.lse, r2.lse)
    # nor do the rows that are masked
    bad = x.clone()
    bad[:100], bad[100:200] = float("nan"), INF
    hidden = torch.where((ids >= 0) & (ids < 200), -INF, offset)
    r2, want = avq.list_log_probs(bad, q, ids, offset=hidden, scale=scale), avq.list_log_probs(x, q, ids, offset=hidden, scale=scale)
    assert torch.equal(r2.logp, want.logp) and torch.equal(r2.lse, want.lse)
    up = normal((nq, m), g)
    got, want = avq.list_log_probs_grad(bad, q, ids, r2.logp, up, scale=scale), avq.list_log_probs_grad(x, q, ids, r2.logp, up, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # +infinity or NaN among a query's scores: no number, and the other queries as before
    if nq > 2:
        for value in (INF, float("nan")):
            bad = offset.clone()
            bad[0, 4], ids[0, 4] = value, 3
            good = avq.list_log_probs(x, q, ids, offset=offset, scale=scale)
            r3 = avq.list_log_probs(x, q, ids, offset=bad, scale=scale)
            real = (ids[0] >= 0) & (ids[0] < 500)
            assert bool(torch.isnan(r3.lse[0])) and bool(torch.isnan(r3.logp[0][real]).all()) and bool((r3.logp[0][~real] == -INF).all())
            assert torch.equal(r3.logp[1:], good.logp[1:]) and torch.equal(r3.lse[1:], good.lse[1:])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("m", [2, 9, 700])
def test_answers_that_are_nearly_certain_keep_their_accuracy(kind, m):
    """-log p = log(1 + sum of the others' e^(s_i - s_t)), whose relative error is that of the scores' differences."""
    g, x, q, ids, _ = inputs(300, 64, 12, m, kind, 5)
    ids = torch.randint(0, 300, (12, m), generator=g, device="cuda", dtype=torch.int32)
    offset = torch.full((12, m), -18.0, device="cuda")
    offset[:, 0] = 0.0
    r = avq.list_log_probs(x, q, ids, offset=offset, scale=0.02)
    s, e, _ = scores(x, q, ids, 0.02, offset)
    away = s[:, 1:] - s[:, :1]
    want = -torch.log1p(torch.exp(away).sum(1))
    size = s.abs().amax(1)
    within(r.logp[:, 0], want, want.abs() * (4 * e.amax(1) + 4 * U * size + (m + 16) * U), "log p of the likeliest")
    # and the gradient of -log p of it is that of 1 - p
    up = torch.zeros((12, m), device="cuda")
    up[:, 0] = -1.0
    do = avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=0.02)[2]
    p = torch.expm1(r.logp[:, 0].double())
    within(do[:, 0], p, p.abs() * 8 * U, "offset's gradient")


def grads(x, q, ids, logp, up, up_lse, scale):
    """dq, dx, G in 64 bits from the given logp, and how far fp32 may be from them."""
    n, (nq, m) = x.shape[0], ids.shape
    s32 = torch.tensor(scale, dtype=torch.float32).item()
    real = (ids >= 0) & (ids < n) & (logp > -INF)
    at = torch.where(real, ids, 0).long()
    g = torch.where(real, up.double(), 0.0)
    p = torch.where(real, logp.double().exp(), 0.0)
    a = g.sum(1, keepdim=True)
    if up_lse is not None:
        a = a - up_lse.double()[:, None]
    G = torch.where(real, g - p * a, 0.0)
    e = (m + 4) * U * p * (g.abs().sum(1, keepdim=True) + (0.0 if up_lse is None else up_lse.double().abs()[:, None])) + 8 * U * (g.abs() + 2 * p * a.abs()) + 1e-37
    e = torch.where(real, e, 0.0)
    rows, qd = x.double()[at], q.double()
    dq = torch.bmm(G[:, None, :], rows)[:, 0] * s32
    e_q = (torch.bmm(e[:, None, :], rows.abs())[:, 0] + (m + 4) * U * torch.bmm(G.abs()[:, None, :], rows.abs())[:, 0]) * abs(s32)
    flat, many = at.reshape(-1), torch.zeros(n, dtype=torch.float64, device="cuda")
    many.index_add_(0, flat, real.double().reshape(-1))

    def spread(w, v):
        return torch.zeros((n, x.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, flat, (w[:, :, None] * v[:, None, :]).reshape(-1, x.shape[1]))

    dx = spread(G, qd) * s32
    e_x = (spread(e, qd.abs()) + (many[:, None] + 4) * U * spread(G.abs(), qd.abs())) * abs(s32)
    return dq, e_q, dx, e_x, G, e


def check_grads(got, x, q, ids, logp, up, up_lse, scale, kind, held=None):
    dq, e_q, dx, e_x, G, e = grads(x, q, ids, logp, up, up_lse, scale)
    within(got[2], G, e, "doffset")
    within(got[0], dq, e_q + HALF[kind] * dq.abs() * 1.01 + TINY[kind], "dqueries")
    if held is not None:
        touched = torch.zeros(x.shape[0], dtype=torch.bool, device="cuda")
        touched[ids[(ids >= 0) & (ids < x.shape[0])].long()] = True
        assert torch.equal(got[1][~touched], held[~touched])
        dx = dx + held.double()
        e_x = e_x + U * dx.abs()
    within(got[1], dx, e_x + HALF[kind] * dx.abs() * 1.01 + TINY[kind], "dpoints")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,nq,m", SHAPES)
def test_list_log_probs_grad(kind, n, d, nq, m):
    g, x, q, ids, scale = inputs(n, d, nq, m, kind, 1)
    offset = normal((nq, m), g)
    if m > 3:
        offset[:, 2] = -INF
    logp = avq.list_log_probs(x, q, ids, offset=offset, scale=scale).logp
    up, up_lse = normal((nq, m), g), normal((nq,), g)
    got = avq.list_log_probs_grad(x, q, ids, logp, up, scale=scale)
    check_grads(got, x, q, ids, logp, up, None, scale, kind)
    again = avq.list_log_probs_grad(x, q, ids, logp, up, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "two calls differ"
    # strided, with the gradient of lse, added to a held gradient; upstream values of padding and masks are not looked at
    held = normal((n, d), g, TYPES[kind])
    out = strided(held, 3, 1)
    up2 = torch.where(logp == -INF, float("nan"), up)
    got = avq.list_log_probs_grad(strided(x, 5, 3), strided(q, 7, 1), ids, logp, up2, grad_lse=up_lse, scale=-scale, out_points=out, accumulate=True)
    assert got[1] is out
    check_grads(got, x, q, ids, logp, up, up_lse, -scale, kind, held)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq,m", [(600, 9), (1500, 9), (40, 9), (4500, 5), (2, 900)])
def test_one_row_in_every_list_and_rows_of_no_weight(kind, nq, m):
    """The gradient of a shared row is the sum over all queries; rows of G = 0 add nothing though they hold NaN."""
    n, d = 50, 100
    g, x, q, _, scale = inputs(n, d, nq, m, kind, 2)
    ids = torch.full((nq, m), 7, dtype=torch.int32, device="cuda")
    ids[:, 1] = 11
    logp = torch.log_softmax(normal((nq, m), g), 1)
    logp[:, 1] = -INF
    up = normal((nq, m), g)
    x[11] = float("nan")
    got = avq.list_log_probs_grad(x, q, ids, logp, up, scale=scale)
    x[11] = 0.0
    check_grads(got, x, q, ids, logp, up, None, scale, kind)
    assert bool((got[1][11] == 0).all())


def test_gradients_against_differences():
    g, x, q, ids, scale = inputs(30, 6, 5, 8, "f32", 3)
    offset = normal((5, 8), g)
    up, up_lse = normal((5, 8), g), normal((5,), g)
    real = (ids >= 0) & (ids < 30)

    def loss(xd, qd, od):
        s = (xd[torch.where(real, ids, 0).long()] * qd[:, None, :]).sum(2) * torch.tensor(scale, dtype=torch.float32).item() + od
        s = torch.where(real, s, -INF)
        lse = torch.logsumexp(s, 1)
        some = lse > -INF
        return (torch.where(real, (s - lse[:, None]) * up.double(), 0.0)).sum() + torch.where(some, lse * up_lse.double(), 0.0).sum()

    r = avq.list_log_probs(x, q, ids, offset=offset, scale=scale)
    got = avq.list_log_probs_grad(x, q, ids, r.logp, up, grad_lse=up_lse, scale=scale)
    base = [x.double(), q.double(), offset.double()]
    for which, grad in ((0, got[1]), (1, got[0]), (2, got[2])):
        for i in range(0, base[which].numel(), 7):
            h = 1e-5
            a, b = [t.clone() for t in base], [t.clone() for t in base]
            a[which].view(-1)[i] += h
            b[which].view(-1)[i] -= h
            slope = (loss(*a) - loss(*b)).item() / (2 * h)
            # the kernel's own bound is a few hundred u of sums below 100, the difference's h^2 times third derivatives
            assert abs(grad.reshape(-1)[i].item() - slope) < 1e-4, (which, i)


@pytest.mark.parametrize("nq,m", [(64, 70), (20, 9), (3, 2500), (300, 80), (4200, 6)])
def test_captured_calls_follow_their_inputs(nq, m):
    """Both calls in a graph, on another stream than the default, replayed over changed inputs with eager work in between."""
    n, d = 3000, 100
    g, x, q, ids, scale = inputs(n, d, nq, m, "f32", 4)
    up = normal((nq, m), g)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        r = avq.list_log_probs(x, q, ids, scale=scale)
        avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=scale)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            r = avq.list_log_probs(x, q, ids, scale=scale)
            held = avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=scale)
    torch.cuda.synchronize()
    for step in range(4):
        x.copy_(normal((n, d), g))
        ids.copy_(lists((nq, m), n, g))
        want = avq.list_log_probs(x, q, ids, scale=scale)
        more = avq.list_log_probs_grad(x, q, ids, want.logp, up, scale=scale)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r.logp, want.logp) and torch.equal(r.lse, want.lse)
        assert all(torch.equal(a, b) for a, b in zip(held, more))


def test_on_another_stream():
    g, x, q, ids, scale = inputs(2000, 128, 30, 40, "bf16", 6)
    want = avq.list_log_probs(x, q, ids, scale=scale)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = avq.list_log_probs(x, q, ids, scale=scale, stream=stream)
    stream.synchronize()
    assert torch.equal(got.logp, want.logp) and torch.equal(got.lse, want.lse)


def test_a_list_of_all_rows_is_the_softmax_over_all_rows():
    g, x, q, _, scale = inputs(400, 60, 20, 1, "f32", 7)
    ids = torch.arange(400, device="cuda", dtype=torch.int32).repeat(20, 1)
    up = normal((20, 400), g)
    a = avq.list_log_probs(x, q, ids, scale=scale)
    b = avq.log_probs(x, q, ids, scale=scale)
    check_probs(a, x, q, ids, scale)
    s, e, _ = scores(x, q, ids, scale, None)
    assert torch.allclose(a.lse, b.lse, rtol=0, atol=2 * (e.max().item() + 500 * U))
    ga = avq.list_log_probs_grad(x, q, ids, a.logp, up, scale=scale)
    gb = avq.log_probs_grad(x, q, ids, b.lse, up, scale=scale)
    # fp32 pairs: 2^-20 of an entry or of the largest, over sums of 400 and 20 terms
    assert torch.allclose(ga[0], gb[0], rtol=1e-4, atol=1e-3) and torch.allclose(ga[1], gb[1], rtol=1e-4, atol=1e-3)


def test_rows_beyond_32_bits():
    """A table of more than 2^32 bytes and 2^31 elements: its last rows are those that are read and get a gradient."""
    n, d = 2_200_000, 1000
    x = torch.zeros((n, d), dtype=torch.float16, device="cuda")
    last = normal((50, d), gen(1), torch.float16)
    x[-50:] = last
    g = gen(2)
    for nq, m in ((3, 40), (60, 70)):
        q, near = normal((nq, d), g, torch.float16), lists((nq, m), 50, g)
        ids = torch.where((near >= 0) & (near < 50), near + (n - 50), near.clamp(max=-1))
        near = torch.where(ids >= 0, near, -1)
        r, want = avq.list_log_probs(x, q, ids, scale=0.1), avq.list_log_probs(last, q, near, scale=0.1)
        assert torch.equal(r.logp, want.logp) and torch.equal(r.lse, want.lse)
        up = normal((nq, m), g)
        got, small = avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=0.1), avq.list_log_probs_grad(last, q, near, r.logp, up, scale=0.1)
        assert torch.equal(got[0], small[0]) and torch.equal(got[2], small[2])
        assert not bool(got[1][: n - 50].any())
        check_grads((got[0], got[1][-50:], got[2]), last, q, near, r.logp, up, None, 0.1, "f16")
        del got


def test_two_streams_at_once():
    """Calls of two streams at the same time have scratch of their own."""
    made = [inputs(4000, 64, 300, 40, "f32", seed) for seed in (8, 9)]
    ups = [normal((300, 40), g) for g, *_ in made]
    want = []
    for (g, x, q, ids, scale), up in zip(made, ups):
        r = avq.list_log_probs(x, q, ids, scale=scale)
        want.append((r, avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=scale)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(5):
        got = []
        for stream, (g, x, q, ids, scale), up in zip(streams, made, ups):
            with torch.cuda.stream(stream):
                r = avq.list_log_probs(x, q, ids, scale=scale)
                got.append((r, avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=scale)))
        torch.cuda.synchronize()
        for (r, grad), (r2, grad2) in zip(got, want):
            assert torch.equal(r.logp, r2.logp) and all(torch.equal(a, b) for a, b in zip(grad, grad2))


def test_either_gradient_alone():
    """The C call's dqueries and dpoints may each be left out."""
    for nq, m in ((20, 9), (90, 70), (3, 2500)):
        g, x, q, ids, scale = inputs(700, 48, nq, m, "f32", 10)
        r = avq.list_log_probs(x, q, ids, scale=scale)
        up = normal((nq, m), g)
        want = avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=scale)
        ws = torch.empty(max(avq.lib().avq_list_log_probs_grad_scratch(700, 48, nq, m), 256), dtype=torch.uint8, device="cuda")
        dq, dx, do = torch.empty_like(q), torch.empty_like(x), torch.empty_like(up)
        for queries, points in ((True, False), (False, True), (False, False)):
            for t in (dq, dx, do):
                t.fill_(7.0)
            assert avq.lib().avq_list_log_probs_grad(x.data_ptr(), 0, 700, 48, 48, q.data_ptr(), nq, 48, scale, ids.data_ptr(), m, r.logp.data_ptr(), up.data_ptr(), None,
                                                      do.data_ptr(), dq.data_ptr() if queries else None, 48, dx.data_ptr() if points else None, 48, 0, ws.data_ptr(), ws.numel(),
                                                      torch.cuda.current_stream().cuda_stream) == 0
            torch.cuda.synchronize()
            assert torch.equal(do, want[2])
            assert torch.equal(dq, want[0]) if queries else bool((dq == 7.0).all())
            assert torch.equal(dx, want[1]) if points else bool((dx == 7.0).all())


# ---- subnormal elements --------------------------------------------------------------------------

# deviations of the rows, of the queries and the scale; most of the rows' elements are subnormal in their type, and decide the scores
SUBNORMAL = {"f32": (2.0 ** -128, 2.0 ** 120, 256.0), "bf16": (2.0 ** -128, 2.0 ** 120, 256.0), "f16": (2.0 ** -16, 2.0 ** 10, 64.0)}


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,nq,m", [(200, 7, 5, 60), (300, 64, 40, 33), (20_000, 101, 4100, 9), (80, 1030, 6, 40), (60, 2050, 3, 30), (30, 4100, 2, 20)])
@pytest.mark.parametrize("swapped", [False, True])
def test_subnormal_elements_count(kind, n, d, nq, m, swapped):
    """Rows (or queries) of subnormal elements: products and sums keep them, as the bound of every other test has it; a flush to zero would make
    all scores 0."""
    g = gen(n + d + nq + m)
    small, large, scale = SUBNORMAL[kind]
    if swapped:
        small, large = large, small
    # (a power of two times normal values in 64 bits, rounded once to the type)
    x = (torch.randn((n, d), generator=g, device="cuda", dtype=torch.float64) * small).to(TYPES[kind])
    q = (torch.randn((nq, d), generator=g, device="cuda", dtype=torch.float64) * large).to(TYPES[kind])
    tiny = q if swapped else x
    least = torch.finfo(TYPES[kind]).smallest_normal
    assert float(((tiny != 0) & (tiny.double().abs() < least)).double().mean()) > 0.5
    ids = lists((nq, m), n, g)
    scale = scale / math.sqrt(d)
    s = scores(x, q, ids, scale, None)[0]
    assert float(s[s > -INF].std()) > 0.5
    r = avq.list_log_probs(x, q, ids, scale=scale)
    check_probs(r, x, q, ids, scale)
    check_probs(avq.list_log_probs(strided(x, 5, 3), strided(q, 7, 1), ids, scale=scale), x, q, ids, scale)
    # (a scale of the gradient's own, so that it stays within the type)
    up, scale = normal((nq, m), g), 0.5 if kind == "f16" else 2.0
    check_grads(avq.list_log_probs_grad(x, q, ids, r.logp, up, scale=scale), x, q, ids, r.logp, up, None, scale, kind)


@pytest.mark.parametrize("kind,d", [("f32", 100), ("bf16", 40), ("f16", 300)])
def test_gradient_of_many_listed_entries(kind, d):
    """More than 4,096 chunks of sorted entries, rows as frequent as words are: listed once or twice, some tens, hundreds, and thousands of times."""
    n, nq, m = 6000, 1501, 150
    g, x, q, _, scale = inputs(n, d, nq, m, kind, 12)
    u = torch.rand((nq, m), generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(n + 1.0)).long() - 1).clamp(0, n - 1).int()
    many = torch.bincount(ids.reshape(-1).long(), minlength=n)
    assert int(((many > 32) & (many < 150)).sum()) > 50 and int((many > 1000).sum()) > 5 and int(((many > 0) & (many < 5)).sum()) > 50
    logp = avq.list_log_probs(x, q, ids, scale=scale).logp
    up = normal((nq, m), g)
    got = avq.list_log_probs_grad(x, q, ids, logp, up, scale=scale)
    check_grads(got, x, q, ids, logp, up, None, scale, kind)
    held = normal((n, d), g, TYPES[kind])
    out = strided(held, 3, 1)
    got = avq.list_log_probs_grad(x, q, ids, logp, up, scale=scale, out_points=out, accumulate=True)
    check_grads(got, x, q, ids, logp, up, None, scale, kind, held)
