"""Operators on rows of learned vectors against plain forms in 64 bits.

Tolerances are bounds, element by element, of what fp32 sums and one rounding to the result's type can be off
(u = 2^-24: a sum of m terms in any order is off by at most m u times the sum of their magnitudes), with the
roundings of G to 16 bits where avq.h states them."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place relative to a value, and the type's smallest step
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-38, "bf16": 1e-38, "f16": 2.0 ** -24}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def random_ids(shape, n, g, padding=0.2):
    ids = torch.randint(0, n, shape, generator=g, device="cuda", dtype=torch.int32)
    draw = torch.rand(shape, generator=g, device="cuda")
    ids = torch.where(draw < padding / 2, -1, ids)
    return torch.where((draw >= padding / 2) & (draw < padding), n + 5, ids)


def within(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    worst = off.max().item() if off.numel() else 0.0
    assert not math.isnan(worst) and worst <= 0, "%s: over the bound by %g" % (what, worst)


def strided(t, extra, shift=0):
    """The same rows inside a wider matrix, starting `shift` elements into it."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, shift:shift + t.shape[1]] = t
    return wide[:, shift:shift + t.shape[1]]


# ---- lookup ----------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,count,scale", [
    (1, 1, 1, 1.0), (10, 3, 0, 2.0), (1000, 100, 7, 1.0), (1000, 100, 513, 10.0), (777, 101, 300, -0.3), (50, 1024, 1000, 32.0), (9, 16384, 5, 1.5),
])
def test_embed(kind, n, d, count, scale):
    g = gen(n + d)
    table, ids = normal((n, d), g, TYPES[kind]), random_ids((count,), n, g)
    real = (ids >= 0) & (ids < n)
    want = (table[torch.where(real, ids, 0).long()].float() * torch.tensor(scale, device="cuda")).to(TYPES[kind])
    want[~real] = 0
    assert torch.equal(avq.embed(table, ids, scale), want)
    wide = strided(torch.zeros((count, d), dtype=TYPES[kind], device="cuda"), 5, 1)
    got = avq.embed(strided(table, 3, 2), ids, scale, out=wide)
    assert got is wide and torch.equal(got, want)


def test_embed_takes_ids_of_any_shape_and_no_nan_of_the_table_for_padding():
    table = torch.full((4, 8), float("nan"), device="cuda")
    table[2] = 1.0
    ids = torch.tensor([[2, -1], [4, 2]], dtype=torch.int32, device="cuda")
    got = avq.embed(table, ids, 3.0)
    assert got.shape == (2, 2, 8)
    assert torch.equal(got[..., 0], torch.tensor([[3.0, 0.0], [0.0, 3.0]], device="cuda"))


def _grad_table(grad, ids, n, scale):
    real = (ids >= 0) & (ids < n)
    at = torch.where(real, ids, 0).long()
    rows = torch.where(real[:, None], grad.double(), 0.0)
    want = torch.zeros((n, grad.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, at, rows)
    mags = torch.zeros_like(want).index_add_(0, at, rows.abs())
    many = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, at, real.double())
    return want * scale, (many[:, None] + 2) * U * mags * abs(scale)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,count,spread", [
    (1, 1, 1, 1), (5, 3, 0, 1), (300, 100, 40, 300), (5000, 100, 4097, 5000), (5000, 101, 2048, 7), (3_000_000, 3, 2500, 3_000_000),
    (100, 64, 20_000, 1), (1000, 1024, 3000, 40), (40, 1030, 333, 40), (70_000, 32, 70_001, 20_000),
])
def test_embed_grad(kind, n, d, count, spread):
    """Ids of `spread` rows only, so that runs of equal ids are short, long, and longer than any part of the work."""
    g = gen(n + d + count)
    grad = normal((count, d), g, TYPES[kind])
    ids = random_ids((count,), spread, g)
    ids = torch.where(ids >= spread, n + 3, ids)
    want, bound = _grad_table(grad, ids, n, 0.7)
    got = avq.embed_grad(grad, ids, n, 0.7)
    within(got, want, bound + HALF[kind] * want.abs() + TINY[kind], "gradient")
    assert torch.equal(got, avq.embed_grad(grad, ids, n, 0.7)), "two calls differ"
    # into a held gradient, strided on both sides
    held = normal((n, d), g, TYPES[kind])
    out = strided(held, 3, 1)
    avq.embed_grad(strided(grad, 2), ids, scale=0.7, out=out, accumulate=True)
    touched = torch.zeros(n, dtype=torch.bool, device="cuda")
    touched[ids[(ids >= 0) & (ids < n)].long()] = True
    want = want + held.double()
    within(out[touched], want[touched], (bound + U * want.abs() + HALF[kind] * want.abs() + TINY[kind])[touched], "sum")
    assert torch.equal(out[~touched], held[~touched])


# ---- layer norm --------------------------------------------------------------------------------

NORM_SHAPES = [(0, 8), (1, 1), (3, 2), (7, 100), (130, 101), (65, 32), (33, 256), (513, 1024), (9, 1030), (5, 2048), (3, 4099), (2, 16384), (2051, 64)]


def _norm_inputs(rows, d, kind):
    g = gen(rows * 31 + d)
    x = (normal((rows, d), g) * 2.0 + 0.5).to(TYPES[kind])
    return g, x, (1.0 + 0.3 * normal((d,), g)).to(TYPES[kind]), normal((d,), g, TYPES[kind])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,d", NORM_SHAPES)
@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm(kind, rows, d, affine):
    eps = 0.1  # (keeps rstd, and with it the bound, small where a row has one or two elements)
    g, x, w, b = _norm_inputs(rows, d, kind)
    if not affine:
        w = b = None
    xd = x.double()
    mean = xd.mean(1) if rows else xd.new_zeros(0)
    var = (xd - mean[:, None]).square().mean(1)
    rstd = (var + eps).rsqrt()
    xhat = (xd - mean[:, None]) * rstd[:, None]
    want = xhat * (w.double() if affine else 1.0) + (b.double() if affine else 0.0)
    top = xd.abs().amax(1) if rows else mean
    e_mean = (d + 2) * U * top                                        # the sum of d terms
    e_rstd = rstd * ((d + 8) * U + 2 * e_mean.square() * rstd.square() + 4 * U + 2 * U * top * rstd)
    for view in (x, strided(x, 3, 1)):
        y, m, r = avq.layer_norm(view, w, b, eps)
        within(m, mean, e_mean, "mean")
        within(r, rstd, e_rstd, "rstd")
        off = (e_mean + U * top)[:, None] * rstd[:, None] + xhat.abs() * (e_rstd / rstd)[:, None] + 4 * U * xhat.abs()
        mag = w.double().abs() if affine else 1.0
        within(y, want, off * mag * 1.01 + 4 * U * want.abs() + HALF[kind] * want.abs() * 1.01 + TINY[kind], "y")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,d", NORM_SHAPES)
@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm_grad(kind, rows, d, affine):
    g, x, w, _ = _norm_inputs(rows, d, kind)
    if not affine:
        w = None
    dy = normal((rows, d), g, TYPES[kind])
    xd, dyd = x.double(), dy.double()
    mean = xd.mean(1).float() if rows else torch.zeros(0, device="cuda")
    rstd = (xd.var(1, unbiased=False) + 0.1).rsqrt().float() if rows else torch.zeros(0, device="cuda")
    m, r = mean.double()[:, None], rstd.double()[:, None]
    xhat = (xd - m) * r
    gg = dyd * (w.double() if affine else 1.0)
    a, c = gg.mean(1, keepdim=True), (gg * xhat).mean(1, keepdim=True)
    want = r * (gg - a - xhat * c)
    e_xhat = 2 * U * (xhat.abs() + xd.abs() * r + m.abs() * r)
    e_a = (d + 2) * U * gg.abs().mean(1, keepdim=True)
    e_c = (d + 4) * U * (gg * xhat).abs().mean(1, keepdim=True) + (gg.abs() * e_xhat).mean(1, keepdim=True)
    size = gg.abs() + a.abs() + (xhat * c).abs()
    bound = r * (e_a + e_c * xhat.abs() + e_xhat * c.abs() + 6 * U * size) * 1.01 + HALF[kind] * want.abs() * 1.01 + TINY[kind]
    want_w, want_b = (dyd * xhat).sum(0), dyd.sum(0)
    bound_w = (rows + 4) * U * (dyd * xhat).abs().sum(0) + (dyd.abs() * e_xhat).sum(0) + HALF[kind] * want_w.abs() * 1.01 + TINY[kind]
    bound_b = (rows + 2) * U * dyd.abs().sum(0) + HALF[kind] * want_b.abs() * 1.01 + TINY[kind]
    first = None
    for up, xs, out in ((dy, x, None), (strided(dy, 5, 2), strided(x, 3, 1), None), (dy.clone(), x, "over grad")):
        dx, dw, db = avq.layer_norm_grad(up, xs, mean, rstd, w, out=up if out else None)
        within(dx, want, bound, "dx")
        within(dw, want_w, bound_w, "dweight")
        within(db, want_b, bound_b, "dbias")
        if first is not None and out:
            assert torch.equal(dx, first[0]) and torch.equal(dw, first[1]) and torch.equal(db, first[2]), "in place differs"
        first = first or (dx, dw, db)


# ---- log probabilities -----------------------------------------------------------------------------

PROB_SHAPES = [
    (1, 1, 1), (5, 3, 2), (31, 32, 16), (33, 100, 17), (1000, 101, 1), (1003, 100, 64), (4097, 130, 65), (20_011, 64, 130), (300, 1024, 300),
    (2049, 1000, 33), (70_001, 16, 5), (515, 5000, 9), (777, 2050, 40), (12_345, 96, 515),
]


def _prob_inputs(n, d, nq, kind, seed=0):
    g = gen(n + 7 * d + 13 * nq + seed)
    x = normal((n, d), g, TYPES[kind])
    q = (normal((nq, d), g) + 0.5 * x[torch.randint(0, n, (nq,), generator=g, device="cuda")].float()).to(TYPES[kind])
    return g, x, q, 2.0 / math.sqrt(d)


def _logits(x, q, scale):
    """Logits in 64 bits and how far fp32 may be from them (products of fp32's accuracy, d + 8 roundings)."""
    xd, qd = x.double(), q.double()
    s32 = torch.tensor(scale, dtype=torch.float32).item()
    return qd @ xd.t() * s32, (d_terms(x) * U * (qd.abs() @ xd.abs().t()) + 1e-30) * abs(s32)


def d_terms(x):
    return x.shape[1] + 8


def _check_probs(r, x, q, scale, ids, k):
    n, nq = x.shape[0], q.shape[0]
    s, e = _logits(x, q, scale)
    lse = torch.logsumexp(s, 1)
    logp = s - lse[:, None]
    p = logp.exp()
    most = e.amax(1)
    # the sum of n terms, each off by its logit's error and a few roundings; and what rounding lse itself costs
    e_lse = most + (n / 64 + 64) * U + 4 * U * lse.abs() + 4 * U * s.abs().amax(1)
    within(r.lse, lse, e_lse, "lse")
    h = -(p * logp).sum(1)
    within(r.entropy, h, e_lse * (2 + (p * logp.abs()).sum(1) + h) + 8 * U * (1 + s.abs().amax(1)) * (1 + h), "entropy")
    if ids is not None:
        rows = ids.reshape(nq, -1)
        real = (rows >= 0) & (rows < n)
        at = torch.where(real, rows, 0).long()
        got = r.logp.reshape(nq, -1)
        assert r.logp.shape == ids.shape and bool((got[~real] == -math.inf).all())
        bound = e.gather(1, at) + e_lse[:, None] + 4 * U * logp.gather(1, at).abs()
        within(got[real], logp.gather(1, at)[real], bound[real], "logp")
    if k:
        alt = r.alt_ids.long()
        assert bool((alt >= 0).all()) and bool((alt < n).all())
        assert all(len(set(row)) == k for row in alt.tolist())
        mine = s.gather(1, alt)
        slack = 2 * e.gather(1, alt) + 2 * most[:, None] + 4 * U * mine.abs()
        within(mine, s.topk(k, dim=1).values, slack, "alternatives")                 # as good as the best k, place by place
        within(r.alt_logp, logp.gather(1, alt), slack + e_lse[:, None] + 4 * U * logp.gather(1, alt).abs(), "alt_logp")
        assert bool((r.alt_logp[:, 1:] <= r.alt_logp[:, :-1]).all())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,nq", PROB_SHAPES)
def test_log_probs(kind, n, d, nq):
    g, x, q, scale = _prob_inputs(n, d, nq, kind)
    k = min(n, 10)
    ids = random_ids((nq, 3), n, g)
    _check_probs(avq.log_probs(x, q, ids, k, scale), x, q, scale, ids, k)
    xs, qs = strided(x, 3, 1), strided(q, 9, 8)
    _check_probs(avq.log_probs(xs, qs, ids[:, 0].contiguous(), 1, -scale), x, q, -scale, ids[:, 0], 1)
    r = avq.log_probs(x, q, scale=scale)
    assert r.logp is None and r.alt_ids is None
    _check_probs(r, x, q, scale, None, 0)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 2])
@pytest.mark.parametrize("n,d", [(1, 7), (31, 3), (32, 64), (33, 8), (2000, 16), (4096, 60), (5000, 100), (777, 128), (3001, 131), (999, 256), (1025, 511), (1500, 1024), (700, 1030), (300, 2048), (100, 4100)])
def test_log_probs_of_one_or_two_queries(kind, nq, n, d):
    g, x, q, scale = _prob_inputs(n, d, nq, kind, 2)
    ids, k = random_ids((nq, 2), n, g), min(n, 6)
    _check_probs(avq.log_probs(x, q, ids, k, scale), x, q, scale, ids, k)
    _check_probs(avq.log_probs(strided(x, 5, 3), strided(q, 1), k=k, scale=-scale), x, q, -scale, None, k)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,nq,k", [(100, 8, 3, 100), (3000, 16, 2, 512), (513, 4, 70, 512), (40_000, 100, 3, 50), (9000, 24, 140, 33), (2100, 40, 300, 7)])
def test_alternatives_are_those_of_lowest_id_among_equals(kind, n, d, nq, k):
    """Rows and queries of small whole numbers: sums are exact, and most scores occur many times."""
    g = gen(n + k)
    x = torch.randint(-2, 3, (n, d), generator=g, device="cuda").to(TYPES[kind])
    q = torch.randint(-2, 3, (nq, d), generator=g, device="cuda").to(TYPES[kind])
    q[0] = 0  # every score the same
    r = avq.log_probs(x, q, k=k, scale=0.25)
    s = q.double() @ x.double().t()
    key = s * n - torch.arange(n, device="cuda").double()
    assert torch.equal(r.alt_ids.long(), key.topk(k, dim=1).indices)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [3, 200])
def test_queries_that_are_not_finite_leave_the_others_alone(kind, nq):
    g, x, q, scale = _prob_inputs(3000, 100, nq, kind)
    good = avq.log_probs(x, q, k=5, scale=scale)
    bad = q.clone()
    bad[1, 7] = float("nan")
    bad[2, 3] = float("inf")
    r = avq.log_probs(x, bad, k=5, scale=scale)
    torch.cuda.synchronize()
    assert bool(torch.isnan(r.lse[1])) and not bool(torch.isfinite(r.lse[2]))
    keep = [i for i in range(nq) if i not in (1, 2)]
    for a, b in ((r.lse, good.lse), (r.entropy, good.entropy), (r.alt_ids, good.alt_ids), (r.alt_logp, good.alt_logp)):
        assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [2, 160])
@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_log_probs_of_rows_of_unequal_size(kind, nq, size):
    """Rows from tiny to large beside one another, logits in the hundreds: sums stay relative to the maximum."""
    g = gen(nq)
    n, d = 2500, 100
    x = normal((n, d), g)
    x = (x * torch.exp(3.0 * normal((n, 1), g)).clamp(max=60.0) * size).to(TYPES[kind])
    q = normal((nq, d), g, TYPES[kind])
    _check_probs(avq.log_probs(x, q, k=3, scale=0.5), x, q, 0.5, None, 3)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 4, 90, 300])
@pytest.mark.parametrize("n,d", [(4000, 475), (20_001, 100)])
def test_log_probability_of_a_row_that_has_nearly_all_of_it(kind, nq, n, d):
    """-log p is the sum of the other rows' e^(s_i - s_t): its relative error is that of the logits' differences, and
    a few roundings of 1 come on top, not of lse."""
    g = gen(nq + n)
    x = normal((n, d), g, TYPES[kind])
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    q = (0.25 * normal((nq, d), g) + 0.9 * x[ids.long()].float()).to(TYPES[kind])
    scale = 25.0 / d
    r = avq.log_probs(x, q, ids, 1, scale)
    s, e = _logits(x, q, scale)
    away = s - s.gather(1, ids.long()[:, None])
    away.scatter_(1, ids.long()[:, None], -math.inf)
    want = -torch.log1p(torch.exp(away).sum(1))
    assert want.max() < 0 and want.median() > -0.1
    bound = want.abs() * (4 * e.amax(1) + 64 * U) + 16 * U
    within(r.logp, want, bound, "logp")
    assert torch.equal(r.alt_ids[:, 0], ids)
    within(r.alt_logp[:, 0], want, bound, "alt_logp")


# ---- their gradient ------------------------------------------------------------------------------------

def _grad_formula(x, q, scale, ids, lse, entropy, up, up_h, up_l, kind):
    """dq and dx in 64 bits, and bounds."""
    n, d = x.shape
    nq = q.shape[0]
    s, e = _logits(x, q, scale)
    logp = s - torch.logsumexp(s, 1)[:, None]
    p = logp.exp()
    h = -(p * logp).sum(1)
    a = torch.zeros(nq, dtype=torch.float64, device="cuda")
    one = torch.zeros((nq, n), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(one)
    if ids is not None:
        rows = ids.reshape(nq, -1)
        real = (rows >= 0) & (rows < n)
        w = torch.where(real, up.reshape(nq, -1).double(), 0.0)
        a = w.sum(1)
        at = torch.where(real, rows, 0).long()
        one.scatter_add_(1, at, w)
        mag.scatter_add_(1, at, w.abs())
    a_mag = mag.sum(1)
    if up_l is not None:
        a, a_mag = a - up_l.double(), a_mag + up_l.double().abs()
    hh = up_h.double() if up_h is not None else torch.zeros_like(a)
    a, a_mag = a + hh * h, a_mag + (hh * h).abs()
    G = one - p * (a[:, None] + hh[:, None] * logp)
    size = mag + p * (a_mag[:, None] + hh.abs()[:, None] * (1 + logp.abs()))
    # p is off by its logit's and lse's error; 16 bits: G is rounded to them
    e_p = e + e.amax(1, keepdim=True) + (n / 64 + 96) * U + 8 * U * (s.abs().amax(1, keepdim=True) + logp.abs())
    e_G = size * (4 * e_p + (ids.numel() // max(nq, 1) + 8 if ids is not None else 8) * U)
    e_G = e_G + {"f32": 2.0 ** -21, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}[kind] * G.abs()
    if kind != "bf16":  # kept relative to the largest upstream gradient (a scale of its own), down to 2^-36 of it
        top = (a_mag + hh.abs() * 30).amax() if nq else 0.0
        e_G = e_G + 2.0 ** -36 * top
    xd, qd = x.double(), q.double()
    s32 = abs(torch.tensor(scale, dtype=torch.float32).item())
    want_q, want_x = G @ xd * scale, G.t() @ qd * scale
    # sums of n (nq) terms; fp32's are kept in parts of at most a few thousand terms
    bound_q = s32 * (e_G @ xd.abs() + (min(n, 4096) + 64) * U * (G.abs() @ xd.abs()))
    bound_x = s32 * (e_G.t() @ qd.abs() + (min(nq, 4096) + 64) * U * (G.abs().t() @ qd.abs()))
    out = lambda w: HALF[kind] * w.abs() * 1.01 + TINY[kind]
    return want_q, bound_q + out(want_q), want_x, bound_x + out(want_x)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,nq", PROB_SHAPES)
@pytest.mark.parametrize("mode", ["loss", "all", "no ids"])
def test_log_probs_grad(kind, n, d, nq, mode):
    g, x, q, scale = _prob_inputs(n, d, nq, kind, 1)
    ids = up = up_h = up_l = None
    if mode == "loss":
        ids, up = random_ids((nq,), n, g), torch.full((nq,), -1.0 / nq, device="cuda")
    elif mode == "all":
        ids = random_ids((nq, 4), min(n, 3), g)  # some of a query's ids are alike
        up, up_h, up_l = normal((nq, 4), g), normal((nq,), g), normal((nq,), g)
    else:
        up_l = normal((nq,), g)
    r = avq.log_probs(x, q, ids, scale=scale)
    want_q, bound_q, want_x, bound_x = _grad_formula(x, q, scale, ids, r.lse, r.entropy, up, up_h, up_l, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h, up_l, scale=scale)
    within(dq, want_q, bound_q, "dqueries")
    within(dx, want_x, bound_x, "dpoints")
    again = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h, up_l, scale=scale)
    assert torch.equal(again[0], dq) and torch.equal(again[1], dx), "two calls differ"
    held = normal((n, d), g, TYPES[kind])
    out = strided(held, 5, 2)
    dq2, got = avq.log_probs_grad(strided(x, 3, 1), strided(q, 9, 8), ids, r.lse, up, r.entropy, up_h, up_l, scale=scale, out_points=out, accumulate=True)
    assert got is out
    within(dq2, want_q, bound_q, "dqueries, strided")
    total = want_x + held.double()
    within(out, total, bound_x + 2 * U * total.abs() + HALF[kind] * total.abs() * 1.01, "dpoints, added")


def test_gradients_agree_with_differences():
    """The whole chain in 64 bits (lookup, layer norm, loss) moved along a random direction, against the operators' gradients."""
    g = gen(5)
    n, d, nq, scale, eps = 700, 36, 50, 0.4, 1e-5
    table, weight, bias = normal((n, d), g), 1 + 0.2 * normal((d,), g), 0.1 * normal((d,), g)
    words, targets = random_ids((nq,), n, g, 0.1), random_ids((nq,), n, g, 0.1)
    real = (targets >= 0) & (targets < n)
    w = torch.where(real, -1.0 / nq, 0.0)

    def loss(t, wt, bs):
        ok = (words >= 0) & (words < n)
        rows = torch.where(ok[:, None], t[torch.where(ok, words, 0).long()] * 3.0, 0.0)
        mean = rows.mean(1, keepdim=True)
        q = (rows - mean) / (rows.var(1, unbiased=False, keepdim=True) + eps).sqrt() * wt + bs
        logp = torch.log_softmax(q @ t.t() * scale, 1)
        h = -(logp.exp() * logp).sum(1)
        return (torch.where(real, logp.gather(1, torch.where(real, targets, 0).long()[:, None])[:, 0], 0.0) * w.double()).sum() + 0.01 * h.sum()

    rows = avq.embed(table, words, 3.0)
    q, mean, rstd = avq.layer_norm(rows, weight, bias, eps)
    r = avq.log_probs(table, q, targets, scale=scale)
    up_h = torch.full((nq,), 0.01, device="cuda")
    dq, dtable = avq.log_probs_grad(table, q, targets, r.lse, w, r.entropy, up_h, scale=scale)
    drows, dweight, dbias = avq.layer_norm_grad(dq, rows, mean, rstd, weight)
    avq.embed_grad(drows, words, scale=3.0, out=dtable, accumulate=True)
    params = [table.double(), weight.double(), bias.double()]
    for i, grad in enumerate((dtable, dweight, dbias)):
        for seed in range(3):
            v = normal(params[i].shape, gen(100 + seed)).double()
            h = 1e-5
            plus, minus = list(params), list(params)
            plus[i], minus[i] = params[i] + h * v, params[i] - h * v
            diff = (loss(*plus) - loss(*minus)).item() / (2 * h)
            mine = (grad.double() * v).sum().item()
            # fp32 gradients: 1e-5 of their size along v; the difference itself: h^2 and 1e-16 / h
            size = (grad.double() * v).abs().sum().item()
            assert abs(diff - mine) <= 1e-5 * size + 1e-6


# ---- streams, graphs, the index ----------------------------------------------------------------------------

def _chain(table, words, targets):
    rows = avq.embed(table, words, 2.0)
    q, mean, rstd = avq.layer_norm(rows)
    r = avq.log_probs(table, q, targets, k=4, scale=0.3)
    w = torch.full((words.numel(),), -0.01, device="cuda")
    dq, dt = avq.log_probs_grad(table, q, targets, r.lse, w, scale=0.3)
    drows, dw, db = avq.layer_norm_grad(dq, rows, mean, rstd)
    avq.embed_grad(drows, words, scale=2.0, out=dt, accumulate=True)
    return [rows, q, r.logp, r.lse, r.entropy, r.alt_ids, r.alt_logp, dt, dw, db]


@pytest.mark.parametrize("kind,count", [("f32", 90), ("bf16", 300)])
def test_chain_on_another_stream_and_in_a_graph(kind, count):
    g = gen(9)
    table = normal((6000, 100), g, TYPES[kind])
    words, targets = random_ids((count,), 6000, g), random_ids((count,), 6000, g)
    want = [t.clone() for t in _chain(table, words, targets)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = avq.embed(table, words, 2.0, stream=side)
    raw = avq.embed(table, words, 2.0, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want[0]) and torch.equal(raw, want[0])
    with torch.cuda.stream(side):
        got = _chain(table, words, targets)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _chain(table, words, targets)
    for turn in range(4):
        for t in held:
            t.zero_()
        eager = _chain(table, words, targets)  # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), "replay %d" % turn


def test_index_gives_probabilities_of_what_a_search_returned():
    g = gen(11)
    n, d, nq = 9000, 32, 20
    x = torch.nn.functional.normalize(normal((n, d), g))
    q = torch.nn.functional.normalize(normal((nq, d), g))
    idx = avq.Index(d, 16, 4, T=0.2, kmeans_iters=4, encode_passes=2)
    with pytest.raises(avq.AvqError):
        idx.log_probs(q)
    idx.train(x)
    idx.encode(x)
    ids, scores = idx.search(q, 10, 100)
    r = idx.log_probs(q, ids, k=10, scale=8.0)
    _check_probs(r, x, q, 8.0, ids, 10)
    same = avq.log_probs(x, q, ids, 10, 8.0)
    assert all(torch.equal(a, b) for a, b in zip(r, same))
    best, _ = idx.brute_force(q, 10)
    assert torch.equal(best, r.alt_ids)


def test_more_than_two_to_the_31_logits_and_elements():
    g = gen(3)
    n, d, nq = 1_200_000, 32, 2000
    x = normal((n, d), g, torch.bfloat16)
    q = normal((nq, d), g, torch.bfloat16)
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    r = avq.log_probs(x, q, ids, 3, 0.3)
    pick = torch.tensor([0, 1, 999, 1998, 1999], device="cuda")
    part = avq.LogProbs(r.logp[pick], r.lse[pick], r.entropy[pick], r.alt_ids[pick], r.alt_logp[pick])
    _check_probs(part, x, q[pick], 0.3, ids[pick], 3)
    # a table of more than 2^31 elements: its last rows
    table = torch.zeros((2_200_000, 1024), dtype=torch.bfloat16, device="cuda")
    table[-1] = 1.0
    table[-2] = 2.0
    ids = torch.tensor([2_199_999, 2_199_998, 5], dtype=torch.int32, device="cuda")
    assert avq.embed(table, ids)[:, 1023].tolist() == [1.0, 2.0, 0.0]
    got = avq.embed_grad(torch.ones((3, 1024), dtype=torch.bfloat16, device="cuda"), ids, out=table, accumulate=True)
    assert got[[2_199_999, 2_199_998, 5, 6], 1000].tolist() == [2.0, 3.0, 1.0, 0.0]
    r = avq.log_probs(table, torch.full((1, 1024), 0.01, dtype=torch.bfloat16, device="cuda"), k=2)
    assert r.alt_ids[0].tolist() == [2_199_998, 2_199_999]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_small_model_learns_and_its_index_answers(dtype):
    from paper_1908_10396_amd import learn

    corpus = learn.Corpus(2000, topic=8, seed=3)
    model = learn.Model(2000, 32, dtype, seed=3)
    # the first step's gradients are those of the formula, in 64 bits
    a, b = corpus.pairs(512)
    table, weight, bias = (p.detach().double().requires_grad_() for p in model.cast())
    x = table[a.long()]
    off = x - x.mean(1, keepdim=True)
    q = off / (off.square().mean(1, keepdim=True) + 1e-5).sqrt() * weight + bias
    loss = -torch.log_softmax(model.scale * (q @ table.t()), 1)[torch.arange(512, device="cuda"), b.long()].mean()
    loss.backward()
    loss = loss.item()
    got = model.gradients(a, b)
    # fp32: sums of at most 2,000 terms, 2^-24 each; bf16: queries, dq and dx are rounded to 8 bits one after the other
    tol = 2e-5 if dtype == torch.float32 else 2e-2
    assert abs(float(got[0]) - loss) <= tol * loss
    for g, want in zip(got[1:], (table.grad, weight.grad, bias.grad)):
        assert float((g.double() - want).norm()) <= tol * float(want.norm())
    first = loss
    for _ in range(150):
        last = float(model.step(*corpus.pairs(512)))
    assert last < 0.7 * first
    idx = learn.index_of(model, 16)
    try:
        ids, logp, p = learn.answer(model, idx, a, 8, 128)
        s = model.scale * (model.queries(a).double() @ model.table.detach().double().t())
        want = torch.log_softmax(s, 1)
        assert float((logp.double() - want.gather(1, ids.long())).abs().max()) <= 1e-4
        assert float((p.entropy.double() + (want.exp() * want).sum(1)).abs().max()) <= 1e-3
        assert float(logp.exp().sum()) >= 0.9 * float(want.exp().topk(8, 1).values.sum())
    finally:
        idx.close()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,d,nq,m", [(70_001, 100, 1, 3), (70_001, 33, 4, 2), (66_000, 64, 8, 5), (1200, 256, 8, 128), (1100, 257, 5, 1), (1000, 512, 3, 7), (999, 513, 2, 2),
                                      (900, 1000, 1, 1024), (700, 1024, 1, 1), (700, 1025, 1, 2), (600, 2048, 1, 1), (601, 2049, 1, 1), (300, 128, 8, 129), (5, 7, 2, 3), (1, 1, 1, 1)])
def test_log_probs_grad_of_a_few_queries(kind, n, d, nq, m):
    g, x, q, scale = _prob_inputs(n, d, nq, kind, 2)
    ids = random_ids((nq, m), n, g, 0.1)
    ids[0, 0] = min(n - 1, 5)
    ids[-1, -1] = min(n - 1, 5 + 65536)
    up, up_h, up_l = normal((nq, m), g), normal((nq,), g), normal((nq,), g)
    r = avq.log_probs(x, q, ids, scale=scale)
    want_q, bound_q, want_x, bound_x = _grad_formula(x, q, scale, ids, r.lse, r.entropy, up, up_h, up_l, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h, up_l, scale=scale)
    within(dq, want_q, bound_q, "dqueries")
    within(dx, want_x, bound_x, "dpoints")
    again = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h, up_l, scale=scale)
    assert torch.equal(again[0], dq) and torch.equal(again[1], dx), "two calls differ"
    held = normal((n, d), g, TYPES[kind])
    out = strided(held, 5, 2)
    dq2, _ = avq.log_probs_grad(strided(x, 3, 1), strided(q, 9, 8), ids, r.lse, up, r.entropy, up_h, up_l, scale=scale, out_points=out, accumulate=True)
    within(dq2, want_q, bound_q, "dqueries, strided")
    total = want_x + held.double()
    within(out, total, bound_x + 2 * U * total.abs() + HALF[kind] * total.abs() * 1.01, "dpoints, added")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 3, 6, 12])
def test_log_probs_grad_of_rows_with_nearly_all_of_the_probability(kind, nq):
    """G of such a row is g (1 - p), a difference of values near 1: the rounding of lse (and of 16 bits elsewhere) is all it is off by."""
    g = gen(nq)
    n, d = 4000, 100
    x = normal((n, d), g, TYPES[kind])
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    q = (0.25 * normal((nq, d), g) + 0.9 * x[ids.long()].float()).to(TYPES[kind])
    up = torch.full((nq,), -1.0 / nq, device="cuda")
    r = avq.log_probs(x, q, ids, scale=0.25)
    want_q, bound_q, want_x, bound_x = _grad_formula(x, q, 0.25, ids, r.lse, r.entropy, up, None, None, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, scale=0.25)
    within(dq, want_q, bound_q, "dqueries")
    within(dx, want_x, bound_x, "dpoints")


@pytest.mark.parametrize("nq", [1, 2, 4, 7])
@pytest.mark.parametrize("n,d", [(4000, 475), (36_249, 250)])
def test_gradient_of_a_few_queries_whose_answer_is_nearly_certain(nq, n, d):
    """G of the given row is g (1 - p), the sum of the other rows' p: its relative error is that of the logits' differences and a few
    roundings of 1, not that of lse; elsewhere G is off by p's relative error, lse's rounding among it."""
    if nq > 2 and d > 256:
        d = 256  # (what a lane holds)
    g = gen(nq + n)
    x = normal((n, d), g)
    ids = torch.randperm(n, generator=g, device="cuda")[:nq].to(torch.int32)
    q = 0.25 * normal((nq, d), g) + 0.9 * x[ids.long()]
    scale = 25.0 / d
    up = torch.full((nq,), -1.0 / nq, device="cuda")
    r = avq.log_probs(x, q, ids, scale=scale)
    s, e = _logits(x, q, scale)
    p = torch.softmax(s, 1)
    at = torch.arange(nq, device="cuda"), ids.long()
    away = s - s[at][:, None]
    away[at] = -math.inf
    rest = torch.exp(away).sum(1)
    rest = rest / (1 + rest)
    G = -p * up.double()[:, None]
    G[at] = up.double() * rest
    off = 4 * e.amax(1, keepdim=True) + 64 * U
    e_G = G.abs() * (off + 2 * U * r.lse.double().abs()[:, None])
    e_G[at] = up.double().abs() * (rest * off[:, 0] + 16 * U)
    s32 = torch.tensor(scale, dtype=torch.float32).item()
    xd, qd = x.double(), q.double()
    want_q, want_x = G @ xd * scale, G.t() @ qd * scale
    bound_q = s32 * (e_G @ xd.abs() + (4096 + 64) * U * (G.abs() @ xd.abs())) + 2 * U * want_q.abs()
    bound_x = s32 * (e_G.t() @ qd.abs() + (nq + 8) * U * (G.abs().t() @ qd.abs())) + 2 * U * want_x.abs()
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, scale=scale)
    within(dx, want_x, bound_x, "dpoints")
    within(dq, want_q, bound_q, "dqueries")
    # an lse of more rows than these is taken as it is
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse + 0.5, up, scale=scale)
    G = up.double()[:, None] * (torch.nn.functional.one_hot(ids.long(), n).double() - p * math.exp(-0.5))
    assert float((dx.double() - G.t() @ qd * scale).norm() / (G.t() @ qd * scale).norm()) < 1e-4
