"""Operators on rows of learned vectors at the ends of their ranges, against plain forms in 64 bits: answers that are nearly certain,
logits in the hundreds, rows and queries of very unequal size or weight, masks of large, lowest and infinite values, parts of a table,
and the largest counts. Tolerances as in test_gpu_rows: bounds of what fp32 sums and roundings can be off."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")

from test_gpu_rows import HALF, TINY, TYPES, U, _check_probs, _grad_formula, gen, normal, random_ids, strided, within  # noqa: E402


def grid(x, kind):
    """Multiples of 1/32 of at most 8 bits: products and sums of a few hundred of them are exact in every type's arithmetic."""
    return ((x * 32.0).round().clamp(-127, 127) / 32.0).to(TYPES[kind])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 5, 90, 300])
def test_log_probability_and_entropy_of_a_sure_answer(kind, nq):
    """-log p = log(1 + r), r the sum of the other rows' e^(s_i - s): off by the exponents' roundings, relative to r, whatever the size
    of r beside 1; only what a lane adds up together with the answer itself, within 32 rows, may be lost beside it."""
    g = gen(nq)
    n, d, scale = 300_001, 64, 0.5
    x = grid(normal((n, d), g), kind)
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    q = grid(0.9 * x[ids.long()].float() + 0.2 * normal((nq, d), g), kind)
    r = avq.log_probs(x, q, ids, 1, scale)
    s = q.double() @ x.double().t() * scale
    away = s - s.gather(1, ids.long()[:, None])
    away.scatter_(1, ids.long()[:, None], -math.inf)
    assert away.max() < -2.0
    e = away.exp()
    rest = e.sum(1)
    far = torch.where(e > 0, away.abs(), 0.0)
    mates = (ids.long()[:, None] // 32 * 32 + torch.arange(32, device="cuda")).clamp(max=n - 1)
    lost = e.gather(1, mates).sum(1)
    off = (e * (6 * U * far + 256 * U)).sum(1) + lost
    want = -torch.log1p(rest)
    assert want.median() > -0.01
    within(r.logp, want, off, "logp")
    assert torch.equal(r.alt_ids[:, 0], ids)
    within(r.alt_logp[:, 0], want, off, "alt_logp")
    h = torch.log1p(rest) + (e * far).sum(1) / (1 + rest)
    within(r.entropy, h, off + (e * far * (6 * U * far + 256 * U)).sum(1) + lost * 1e-2, "entropy")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [9, 33, 65, 257])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradients_of_logits_in_the_hundreds(kind, nq, entropy):
    """The last query's logits are the largest, up to some 400: what the tiles hold past it must not show."""
    g = gen(nq)
    n, d = 700, 100
    x = normal((n, d), g, TYPES[kind])
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    q = normal((nq, d), g) + 1.5 * x[ids.long()].float()
    q[-1] = 4.0 * x[11].float()
    q = q.to(TYPES[kind])
    up, up_h = normal((nq,), g), normal((nq,), g) if entropy else None
    r = avq.log_probs(x, q, ids)
    assert (q[-1].float() @ x[11].float()).item() > 200
    want_q, bound_q, want_x, bound_x = _grad_formula(x, q, 1.0, ids, r.lse, r.entropy, up, up_h, None, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h)
    # (probabilities and entries of G below the normal range, 2^-126, may be taken as 0: that, and there |log p| < 90, for every summand)
    flushed = 2.0 ** -126 * (1 + up.abs().max().item() + (0.0 if up_h is None else 90 * up_h.abs().max().item()))
    within(dx, want_x, bound_x + flushed * (1 + q.double().abs()).sum(0), "dpoints")
    within(dq, want_q, bound_q + flushed * (1 + x.double().abs()).sum(0), "dqueries")


@pytest.mark.parametrize("kind,nq", [("f32", 1), ("f32", 3), ("f32", 64), ("bf16", 1), ("bf16", 3), ("bf16", 64), ("bf16", 65), ("bf16", 300)])
@pytest.mark.parametrize("value", [-1e7, -1e12, -1e30])
def test_log_probs_of_rows_behind_thousands_of_large_masks(kind, nq, value):
    """Logits so large that the rounding of the first maxima, which are masks, is no small exponent."""
    g = gen(nq)
    n, d, k, scale = 5000, 32, 4, 0.3
    x, q = normal((n, d), g), normal((nq, d), g)
    masked = torch.arange(n, device="cuda") < 2500
    x[masked] = 0.0
    x[:, -1] = torch.where(masked, value, 0.0)
    q[:, -1] = 1.0
    x, q = x.to(TYPES[kind]), q.to(TYPES[kind])
    r = avq.log_probs(x, q, k=k, scale=scale)
    assert not bool(masked[r.alt_ids.long()].any())
    part = avq.LogProbs(None, r.lse, r.entropy, r.alt_ids - 2500, r.alt_logp)
    _check_probs(part, x[2500:], q, scale, None, k)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("nq", [1, 5, 80])
def test_log_probs_of_logits_of_a_hundred_million(kind, nq):
    """log p of the largest is 0 and the others' the logits' differences, whatever a logit's own rounding is."""
    g = gen(nq)
    n, d = 2000, 32
    x = torch.randint(-8, 9, (n, d), generator=g, device="cuda").to(TYPES[kind])
    q = torch.randint(-8, 9, (nq, d), generator=g, device="cuda").to(TYPES[kind])
    scale = 2.0 ** 18
    r = avq.log_probs(x, q, k=3, scale=scale)
    s = q.double() @ x.double().t()
    best = s.topk(3, dim=1).values
    count = (s == best[:, :1]).double().sum(1)
    within(r.alt_logp, (best - best[:, :1]) * scale - count.log()[:, None], ((best[:, :1] - best) * scale + 1) * 8 * U, "alt_logp")
    within(r.lse, best[:, 0] * scale + count.log(), (best[:, 0].abs() * scale + 1) * 4 * U, "lse")
    within(r.entropy, count.log(), torch.full_like(count, 64 * U), "entropy")


def _masked(n, d, nq, kind, value, g, share=0.5):
    """Rows whose last element is 0, or for some the mask's value; queries whose last element is 1."""
    x = normal((n, d), g)
    masked = torch.rand((n,), generator=g, device="cuda") < share
    masked[3], masked[n - 1] = True, False
    x[:, -1] = torch.where(masked, value, 0.0)
    q = normal((nq, d), g)
    q[:, -1] = 1.0
    return x.to(TYPES[kind]), q.to(TYPES[kind]), masked


def _without(r, masked, ids, k):
    """The results as those of the rows without a mask: their ids among those."""
    place = torch.where(masked, -1, torch.cumsum(~masked, 0) - 1).int()
    alt = None
    if k:
        assert not bool(masked[r.alt_ids.long()].any()), "a masked alternative"
        alt = place[r.alt_ids.long()]
    real = (ids >= 0) & (ids < masked.numel())
    return avq.LogProbs(r.logp, r.lse, r.entropy, alt, r.alt_logp), torch.where(real, place[torch.where(real, ids, 0).long()], -1)


@pytest.mark.parametrize("kind,value", [("f32", -2.0 ** 24), ("f32", -1e9), ("f32", -1e12), ("f32", -1e30), ("bf16", -1e9), ("bf16", -1e30)])
@pytest.mark.parametrize("nq", [1, 3, 64, 65, 300])
@pytest.mark.parametrize("share", [0.0, 0.5])
def test_log_probs_beside_rows_of_large_masks(kind, value, nq, share):
    """A mask's value in some rows (or in one) costs the others nothing: their bound knows nothing of it."""
    g = gen(nq)
    n, d, k, scale = 3001, 100, 5, 0.3
    x, q, masked = _masked(n, d, nq, kind, value, g, share)
    ids = random_ids((nq, 3), n, g)
    ids = torch.where((ids >= 0) & (ids < n) & masked[ids.clamp(0, n - 1).long()], n - 1, ids)
    r, place = _without(avq.log_probs(x, q, ids, k, scale), masked, ids, k)
    _check_probs(r, x[~masked], q, scale, place, k)
    r = avq.log_probs(x, q, torch.full((nq,), 3, dtype=torch.int32, device="cuda"), 0, scale)
    s = q.double() @ x[3].double() * scale
    within(r.logp, s - r.lse.double(), s.abs() * 256 * U, "logp of a masked row")


@pytest.mark.parametrize("nq", [65, 300])
@pytest.mark.parametrize("value", [-1e7, -1e12, -1e30])
def test_log_probs_of_fp32_rows_behind_thousands_of_large_masks(nq, value):
    test_log_probs_of_rows_behind_thousands_of_large_masks("f32", nq, value)


@pytest.mark.parametrize("kind,value", [("f32", -2.0 ** 24), ("f32", -1e9), ("f32", -1e30), ("bf16", -1e9)])
@pytest.mark.parametrize("nq", [2, 12, 65, 300])
def test_gradients_beside_rows_of_large_masks(kind, value, nq):
    g = gen(nq + 1)
    n, d, scale = 3001, 100, 0.3
    x, q, masked = _masked(n, d, nq, kind, value, g)
    ids = random_ids((nq,), n, g)
    ids = torch.where((ids >= 0) & (ids < n) & masked[ids.clamp(0, n - 1).long()], n - 1, ids)
    up, up_h = normal((nq,), g), normal((nq,), g)
    r = avq.log_probs(x, q, ids, scale=scale)
    _, place = _without(r, masked, ids, 0)
    want_q, bound_q, want_x, bound_x = _grad_formula(x[~masked], q, scale, place, r.lse, r.entropy, up, up_h, None, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h, scale=scale)
    within(dx[~masked], want_x, bound_x, "dpoints")
    assert not bool(dx[masked].any())
    within(dq, want_q, bound_q, "dqueries")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [70, 300])
@pytest.mark.parametrize("rows,queries", [(10, 0), (0, 10), (22, 0), (0, 22), (22, 22)])
def test_rows_and_queries_of_unequal_size(kind, nq, rows, queries):
    """Sizes down to 2^-rows and 2^-queries of the largest."""
    if kind == "f16" and max(rows, queries) > 10:
        pytest.skip("beyond the range of f16")
    g = gen(nq + rows + 2 * queries)
    n, d, scale = 2500, 100, 0.2
    x = normal((n, d), g) * torch.exp2(-rows * torch.rand((n, 1), generator=g, device="cuda"))
    q = normal((nq, d), g) * torch.exp2(-queries * torch.rand((nq, 1), generator=g, device="cuda"))
    x, q = x.to(TYPES[kind]), q.to(TYPES[kind])
    ids = random_ids((nq,), n, g)
    up, up_h = normal((nq,), g), normal((nq,), g)
    r = avq.log_probs(x, q, ids, 3, scale)
    _check_probs(r, x, q, scale, ids, 3)
    want_q, bound_q, want_x, bound_x = _grad_formula(x, q, scale, ids, r.lse, r.entropy, up, up_h, None, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h, scale=scale)
    within(dx, want_x, bound_x, "dpoints")
    within(dq, want_q, bound_q, "dqueries")
    # rows and results apart, added to what is there, the other sign
    r = avq.log_probs(x, q, ids, scale=-scale)
    want_q, bound_q, want_x, bound_x = _grad_formula(x, q, -scale, ids, r.lse, r.entropy, up, up_h, None, kind)
    held = want_x.abs().amax(1, keepdim=True).expand(n, d).to(TYPES[kind])
    out = strided(held, 5, 2)
    dq, dx = avq.log_probs_grad(strided(x, 3, 1), strided(q, 9, 8), ids, r.lse, up, r.entropy, up_h, scale=-scale, out_points=out, accumulate=True)
    total = want_x + held.double()
    within(dx, total, bound_x + 2 * U * total.abs() + HALF[kind] * total.abs() * 1.01, "dpoints, added")
    within(dq, want_q, bound_q, "dqueries, strided")


@pytest.mark.parametrize("value", [-2.0, -1e9, -math.inf])
def test_gradients_beside_masks_in_several_parts_of_the_rows(value):
    """So many queries that the rows are taken in parts; the given rows lie in all of them."""
    g = gen(8)
    n, d, nq, scale = 13_000, 16, 40_000, 0.5
    x, q, masked = _masked(n, d, nq, "f32", value, g)
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    ids = torch.where(masked[ids.long()], n - 1, ids)
    up = normal((nq,), g)
    r = avq.log_probs(x, q, ids, scale=scale)
    keep, place = slice(None), ids
    if value < -1e3:
        keep = ~masked
        _, place = _without(r, masked, ids, 0)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, scale=scale)
    want_q, bound_q, want_x, bound_x = _grad_formula(x[keep], q, scale, place, r.lse, r.entropy, up, None, None, "f32")
    within(dx[keep], want_x, bound_x, "dpoints")
    within(dq[:, :-1], want_q[:, :-1], bound_q[:, :-1], "dqueries")
    if value < -1e3:
        assert not bool(dx[masked].any())


def _gradient_of_weighted(x, q, scale, ids, up, kind):
    """The gradient of the loss in 64 bits; bounds as in _grad_formula, but what G is kept down to is relative to its own query's
    upstream gradient."""
    n = x.shape[0]
    xd, qd = x.double(), q.double()
    s32 = abs(torch.tensor(scale, dtype=torch.float32).item())
    s = qd @ xd.t() * s32
    e = ((x.shape[1] + 8) * U * (qd.abs() @ xd.abs().t()) + 1e-30) * s32
    logp = s - torch.logsumexp(s, 1)[:, None]
    w = up.double()[:, None]
    one = torch.nn.functional.one_hot(ids.long(), n).double()
    G = w * (one - logp.exp())
    e_p = e + e.amax(1, keepdim=True) + (n / 64 + 96) * U + 8 * U * (s.abs().amax(1, keepdim=True) + logp.abs())
    e_G = w.abs() * (one + logp.exp()) * (4 * e_p + 16 * U) + {"f32": 2.0 ** -21, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}[kind] * G.abs()
    if kind != "bf16":
        e_G = e_G + 2.0 ** -36 * w.abs()
    want_q, want_x = G @ xd * scale, G.t() @ qd * scale
    bound_q = s32 * (e_G @ xd.abs() + (min(n, 4096) + 64) * U * (G.abs() @ xd.abs()))
    bound_x = s32 * (e_G.t() @ qd.abs() + (q.shape[0] + 64) * U * (G.abs().t() @ qd.abs()))
    return want_q, bound_q + HALF[kind] * want_q.abs() * 1.01 + TINY[kind], want_x, bound_x + HALF[kind] * want_x.abs() * 1.01 + TINY[kind]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [7, 33, 70, 300])
@pytest.mark.parametrize("least", [1e-4, 1e-8])
def test_gradients_of_queries_of_unequal_weight(kind, nq, least):
    """Upstream gradients between `least` and 1: each query's gradient is as exact as if it were alone."""
    g = gen(nq)
    n, d, scale = 20_000, 64, 0.25
    x, q = normal((n, d), g, TYPES[kind]), normal((nq, d), g, TYPES[kind])
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    up = -torch.exp(math.log(least) * torch.rand((nq,), generator=g, device="cuda"))
    up[0], up[-1] = -1.0, -least
    r = avq.log_probs(x, q, ids, scale=scale)
    # results large enough for their type: a common power of two, which changes no bound but by itself
    up = up * 2.0 ** 12
    want_q, bound_q, want_x, bound_x = _gradient_of_weighted(x, q, scale, ids, up, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, scale=scale)
    within(dq, want_q, bound_q, "dqueries")
    within(dx, want_x, bound_x, "dpoints")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [33, 70])
def test_queries_without_upstream_gradient_beside_others(kind, nq):
    g = gen(nq)
    n, d, scale = 3000, 64, 0.25
    x, q = normal((n, d), g, TYPES[kind]), normal((nq, d), g, TYPES[kind])
    ids = torch.randint(0, n, (nq,), generator=g, device="cuda", dtype=torch.int32)
    up = torch.where(torch.arange(nq, device="cuda") % 3 == 0, 0.0, 1e-3)
    r = avq.log_probs(x, q, ids, scale=scale)
    want_q, bound_q, want_x, bound_x = _gradient_of_weighted(x, q, scale, ids, up, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, scale=scale)
    within(dq, want_q, bound_q, "dqueries")
    within(dx, want_x, bound_x, "dpoints")
    assert not bool(dq[::3].any())
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, torch.zeros_like(up), scale=scale)
    assert not bool(dq.any()) and not bool(dx.any())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [12, 21, 77, 300])
def test_gradient_of_given_rows_under_weights_that_are_alike(kind, nq):
    """With the gradients of log p and of lse the same, G is g at the given row alone, -1 / nq: 16 bits hold it relative to the largest, so
    that nothing but the results' own rounding is left."""
    g = gen(nq)
    n, d, scale = 900, 64, 0.25
    x, q = normal((n, d), g, TYPES[kind]), normal((nq, d), g, TYPES[kind])
    ids = torch.randperm(n, generator=g, device="cuda")[:nq].to(torch.int32)  # (no row is given twice)
    up = torch.full((nq,), -1.0 / nq, device="cuda")
    r = avq.log_probs(x, q, ids, scale=scale)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, grad_lse=up, scale=scale)
    want_q, want_x = up.double()[:, None] * x[ids.long()].double() * scale, up.double()[:, None] * q.double() * scale
    # fp32 beyond a few queries: pairs, 2^-21 of a product
    bound = HALF[kind] * 1.01 + (2.0 ** -20 if kind == "f32" else 8 * U)
    within(dq, want_q, bound * want_q.abs() + TINY[kind], "dqueries")
    within(dx[ids.long()], want_x, bound * want_x.abs() + TINY[kind], "dpoints")


@pytest.mark.parametrize("nq", [12, 65, 300])
def test_fp32_rows_a_little_within_the_spread_of_one_scale(nq):
    """Rows 2^-14.5 of the table's largest, which has no probability: they are all that the queries' gradient is of."""
    test_gradients_beside_rows_of_large_masks("f32", -(2.0 ** 16), nq)
    test_log_probs_beside_rows_of_large_masks("f32", -(2.0 ** 16), nq, 0.5)
    test_log_probs_beside_rows_of_large_masks("f32", -512.0, nq, 0.5)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [24, 130])
@pytest.mark.parametrize("weight", [2.0 ** -15, 2.0 ** -20])
def test_rows_that_only_queries_of_little_weight_reach(kind, nq, weight):
    """Half of the rows are reached by half of the queries (logits 200 apart), whose upstream gradients are `weight` of the others'."""
    g = gen(nq)
    n, d = 1000, 32
    x, q = 0.5 * normal((n, d), g), 0.5 * normal((nq, d), g)
    x[:, :2] = 0.0
    x[: n // 2, 0], x[n // 2:, 1] = 10.0, 10.0
    sign = torch.where(torch.arange(nq, device="cuda") % 2 == 0, 10.0, -10.0)
    q[:, 0], q[:, 1] = sign, -sign
    x, q = x.to(TYPES[kind]), q.to(TYPES[kind])
    ids = torch.randint(0, n // 2, (nq,), generator=g, device="cuda", dtype=torch.int32) + torch.where(sign > 0, 0, n // 2).int()
    up = torch.where(sign > 0, 1.0, weight) * 2.0 ** 8
    r = avq.log_probs(x, q, ids)
    want_q, bound_q, want_x, bound_x = _gradient_of_weighted(x, q, 1.0, ids, up, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up)
    within(dx[n // 2:], want_x[n // 2:], bound_x[n // 2:], "dpoints of little weight")
    within(dx[: n // 2], want_x[: n // 2], bound_x[: n // 2], "dpoints")
    within(dq, want_q, bound_q, "dqueries")


@pytest.mark.parametrize("nq", [1, 2, 4, 7])
@pytest.mark.parametrize("other", [2e-5, 5e-5, 1e-3])
def test_gradient_of_a_part_of_a_table_whose_other_part_is_unlikely(nq, other):
    """lse of a whole table, of which these rows lack a probability `other`: G of the given row is g (1 - p), p that of the whole
    table, to what lse's rounding (2^-24 of it, of these rows' and of the whole's) and some roundings of 1 leave."""
    g = gen(nq)
    n, d = 4000, 250
    x = normal((n, d), g)
    ids = torch.randperm(n, generator=g, device="cuda")[:nq].to(torch.int32)
    q = 0.25 * normal((nq, d), g) + 0.9 * x[ids.long()]
    scale = 25.0 / d
    up = torch.full((nq,), -1.0 / nq, device="cuda")
    s = q.double() @ x.double().t() * torch.tensor(scale, dtype=torch.float32).item()
    r = avq.log_probs(x, q, ids, scale=scale)  # (these rows' lse has the products' own errors, which are no part of 1 - p)
    whole = r.lse.double() - math.log1p(-other)
    dq, dx = avq.log_probs_grad(x, q, ids, whole.float(), up, scale=scale)
    at = torch.arange(nq, device="cuda"), ids.long()
    p = torch.softmax(s, 1) * (1 - other)
    given = up.double() * (1 - p[at])
    off = up.double().abs() * (2 * U * whole.abs() + 32 * U)
    # the given rows' gradient along their query: G of that row times |q|^2, and the other queries' small shares
    G = -p * up.double()[:, None]
    G[at] = given
    want = (G.t() @ q.double() * scale)[ids.long()]
    bound = off[:, None] * q.double().abs() * scale + 1e-4 * (G.abs().t() @ q.double().abs() * scale)[ids.long()]
    within(dx[ids.long()], want, bound, "dpoints of the given rows")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 2, 5, 64, 65, 300])
@pytest.mark.parametrize("value", ["infinite", "lowest"])
@pytest.mark.parametrize("sign", [1, -1])
def test_log_probs_beside_rows_of_infinite_and_lowest_masks(kind, nq, value, sign):
    """Logits of -infinity are a probability of 0: lse, entropy and the alternatives are those of the other rows."""
    g = gen(nq)
    n, d, k, scale = 3001, 100, 5, 0.3 * sign
    value = -sign * (math.inf if value == "infinite" else torch.finfo(TYPES[kind]).max)
    x, q, masked = _masked(n, d, nq, kind, value, g)
    ids = random_ids((nq, 3), n, g)
    ids = torch.where((ids >= 0) & (ids < n) & masked[ids.clamp(0, n - 1).long()], n - 1, ids)
    r, place = _without(avq.log_probs(x, q, ids, k, scale), masked, ids, k)
    _check_probs(r, x[~masked], q, scale, place, k)
    r = avq.log_probs(x, q, torch.full((nq,), 3, dtype=torch.int32, device="cuda"), 0, scale)
    s = q.double() @ x[3].double() * scale
    if math.isinf(value):
        assert bool((r.logp == -math.inf).all())
    else:
        within(r.logp, s - r.lse.double(), s.abs() * 256 * U, "logp of a masked row")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 5, 70])
def test_rows_that_are_not_finite_show(kind, nq):
    """NaN, +infinity, and infinity times zero in any row: no query's sum is a number."""
    g = gen(nq)
    x, q, _ = _masked(3001, 100, nq, kind, 0.0, g)
    for value, at in ((float("nan"), 5), (math.inf, 99), (-math.inf, 7)):
        bad = x.clone()
        bad[1234, at] = value
        if at == 7:
            q = q.clone()
            q[:, 7] = 0.0
        r = avq.log_probs(bad, q, k=2, scale=0.3)
        assert not bool(torch.isfinite(r.lse).any())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 3, 70, 300])
def test_alternatives_where_there_are_fewer_rows_than_asked_for_without_a_mask(kind, nq):
    """The masked rows come last, by their ids; a query with all rows masked has them all so."""
    g = gen(nq)
    n, d = 130, 40
    x, q, masked = _masked(n, d, nq, kind, -math.inf, g)
    r = avq.log_probs(x, q, k=n)
    good = int((~masked).sum())
    assert torch.equal(torch.sort(r.alt_ids[:, :good], 1).values.long(), torch.nonzero(~masked)[:, 0].expand(nq, good))
    assert torch.equal(r.alt_ids[:, good:].long(), torch.nonzero(masked)[:, 0].expand(nq, n - good))
    assert bool(torch.isfinite(r.alt_logp[:, :good]).all()) and bool((r.alt_logp[:, good:] == -math.inf).all())
    x[:, -1] = -math.inf
    r = avq.log_probs(x, q, k=n)
    assert bool((r.lse == -math.inf).all())
    assert torch.equal(r.alt_ids.long(), torch.arange(n, device="cuda").expand(nq, n))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nq", [1, 2, 3, 7, 12, 65, 300])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradients_beside_rows_of_infinite_masks(kind, nq, entropy):
    """Rows of probability 0 get no gradient; the queries' is that of the other rows, but in the mask's own column, where it is 0 times
    infinity."""
    g = gen(nq)
    n, d, scale = 3001, 100, 0.3
    x, q, masked = _masked(n, d, nq, kind, -math.inf, g)
    ids = random_ids((nq,), n, g)
    ids = torch.where((ids >= 0) & (ids < n) & masked[ids.clamp(0, n - 1).long()], n - 1, ids)
    up, up_h = normal((nq,), g), normal((nq,), g) if entropy else None
    r = avq.log_probs(x, q, ids, scale=scale)
    _, place = _without(r, masked, ids, 0)
    want_q, bound_q, want_x, bound_x = _grad_formula(x[~masked], q, scale, place, r.lse, r.entropy, up, up_h, None, kind)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, r.entropy, up_h, scale=scale)
    within(dx[~masked], want_x, bound_x, "dpoints")
    assert not bool(dx[masked].any())
    within(dq[:, :-1], want_q[:, :-1], bound_q[:, :-1], "dqueries")


def test_gradient_of_as_many_given_ids_as_there_can_be_threads():
    g = gen(1)
    n, d, nq, m = 64, 8, 1 << 16, 1 << 10
    x, q = normal((n, d), g), normal((nq, d), g)
    ids = torch.full((nq, m), -1, dtype=torch.int32, device="cuda")
    ids[:, 5], ids[:, m - 1] = 3, 9
    ids[7, ::2] = 3
    up = torch.zeros((nq, m), device="cuda")
    up[:, 5], up[:, m - 1] = 0.5, -1.0
    up[7, ::2] = 2.0 ** -9
    up[7, 5] = 0.0
    ids[7, 5] = -1
    r = avq.log_probs(x, q, scale=0.3)
    dq, dx = avq.log_probs_grad(x, q, ids, r.lse, up, scale=0.3)
    two = torch.tensor([[3, 9]], dtype=torch.int32, device="cuda").expand(nq, 2).contiguous()
    up2 = torch.tensor([[0.5, -1.0]], device="cuda").expand(nq, 2).contiguous()
    up2[7, 0] = 1.0
    want_q, bound_q, want_x, bound_x = _grad_formula(x, q, 0.3, two, r.lse, None, up2, None, None, "f32")
    within(dq, want_q, bound_q, "dqueries")
    within(dx, want_x, bound_x, "dpoints")


def test_gradient_of_as_many_rows_as_can_be_looked_up():
    g = gen(2)
    count, n = 1 << 28, 1000
    ids = torch.randint(-1, n, (count,), generator=g, device="cuda", dtype=torch.int32)
    grad = torch.ones((count, 1), device="cuda")
    got = avq.embed_grad(grad, ids, n)
    want = torch.bincount((ids + 1).long(), minlength=n + 1)[1:]
    assert torch.equal(got[:, 0].double(), want.double())  # (whole numbers below 2^24: every sum is exact)


def test_many_queries_are_taken_in_parts():
    g = gen(4)
    n, d, nq = 4_200_000, 8, 2_200
    x, q = normal((n, d), g), normal((nq, d), g)
    ids = random_ids((nq, 2), n, g)
    assert avq.lib().avq_log_probs_scratch(0, n, d, nq, 2, 3) < 3 << 29
    r = avq.log_probs(x, q, ids, 3, 0.7)
    pick = torch.tensor([0, 63, 64, 1099, 1100, 1151, 1152, 2198, 2199], device="cuda")
    part = avq.LogProbs(r.logp[pick], r.lse[pick], r.entropy[pick], r.alt_ids[pick], r.alt_logp[pick])
    _check_probs(part, x, q[pick], 0.7, ids[pick], 3)
    for a, b in ((0, 1000), (1000, nq)):  # the whole call against its halves
        half = avq.log_probs(x, q[a:b], ids[a:b].contiguous(), 3, 0.7)
        real = torch.isfinite(half.logp)
        assert torch.equal(torch.isfinite(r.logp[a:b]), real)
        for u, v in ((r.lse[a:b], half.lse), (r.entropy[a:b], half.entropy), (r.logp[a:b][real], half.logp[real])):
            assert float((u - v).abs().max()) <= 1e-4
        assert float((r.alt_logp[a:b] - half.alt_logp).abs().max()) <= 1e-4
