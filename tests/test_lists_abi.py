"""What the operators on lists of rows and the losses refuse, before any pointer reaches the GPU."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")


def f32(*shape):
    return torch.zeros(shape)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def flag(*shape):
    return torch.zeros(shape, dtype=torch.bool)


@pytest.mark.parametrize("call", [
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 9), i32(3, 4)),
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8), i32(3)),                                   # lists have two dimensions
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8), i32(2, 4)),
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8), i32(3, 4), offset=f32(3, 5)),
    lambda: avq.list_log_probs(f32(8, 10).t(), f32(3, 8), i32(3, 4)),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 3), f32(3, 4)),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4), f32(3, 5)),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), None, f32(3, 4)),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4), None),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4), f32(3, 4), grad_lse=f32(4)),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4), f32(3, 4), accumulate=True),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4), f32(3, 4), out_points=f32(9, 8)),
    lambda: avq.distill_loss(f32(3, 4), f32(3, 5)),
    lambda: avq.distill_loss(f32(12), f32(3, 4)),
    lambda: avq.distill_loss(f32(3, 4), f32(3, 4), f32(4)),
    lambda: avq.distill_loss(f32(4, 3).t(), f32(3, 4)),
    lambda: avq.distill_loss_grad(f32(3, 4), f32(3, 4), None),
    lambda: avq.distill_loss_grad(f32(3, 4), f32(3, 4), f32(4)),
    lambda: avq.preference_loss(f32(9), i32(4)),                                                 # three sequences
    lambda: avq.preference_loss(f32(9), i32(0)),
    lambda: avq.preference_loss(f32(9, 1), i32(3)),
    lambda: avq.preference_loss(f32(9), i32(3), ref=f32(8)),
    lambda: avq.preference_loss(f32(9), i32(3), mask=flag(8)),
    lambda: avq.preference_loss_grad(f32(9), i32(3), f32(2)),
    lambda: avq.preference_loss_grad(f32(9), i32(3), None),
    lambda: avq.policy_loss(f32(9), f32(8), f32(2), i32(3)),
    lambda: avq.policy_loss(f32(9), None, f32(2), i32(3)),
    lambda: avq.policy_loss(f32(9), f32(9), f32(3), i32(3)),
    lambda: avq.policy_loss(f32(9), f32(9), f32(9), i32(3), each=False),
    lambda: avq.policy_loss(f32(9), f32(9), f32(2), i32(3), each=True),
    lambda: avq.policy_loss_grad(f32(9), f32(9), f32(2), i32(3), f32(3)),
    lambda: avq.policy_loss_grad(f32(9), f32(9), f32(2), i32(3), None),
])
def test_shapes(call):
    with pytest.raises(ValueError):
        call()


@pytest.mark.parametrize("call", [
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8).half(), i32(3, 4)),
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8), i32(3, 4).long()),
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8), i32(3, 8)[:, ::2]),
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8), i32(3, 4), offset=f32(3, 4).half()),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4).double(), f32(3, 4)),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4), f32(3, 4), out_points=f32(10, 8).half()),
    lambda: avq.distill_loss(f32(3, 4).half(), f32(3, 4)),
    lambda: avq.distill_loss(f32(3, 4), f32(3, 4).double()),
    lambda: avq.distill_loss(f32(3, 4), f32(3, 4), f32(3).half()),
    lambda: avq.preference_loss(f32(9), i32(3).long()),
    lambda: avq.preference_loss(f32(9), i32(3), mask=f32(9)),
    lambda: avq.preference_loss(f32(9).half(), i32(3)),
    lambda: avq.policy_loss(f32(9), f32(9).half(), f32(2), i32(3)),
    lambda: avq.policy_loss(f32(9), f32(9), f32(2).half(), i32(3)),
    # right shapes and types, but on the host
    lambda: avq.list_log_probs(f32(10, 8), f32(3, 8), i32(3, 4)),
    lambda: avq.list_log_probs_grad(f32(10, 8), f32(3, 8), i32(3, 4), f32(3, 4), f32(3, 4)),
    lambda: avq.distill_loss(f32(3, 4), f32(3, 4)),
    lambda: avq.preference_loss(f32(9), i32(3)),
    lambda: avq.policy_loss(f32(9), f32(9), f32(2), i32(3)),
])
def test_types_and_devices(call):
    with pytest.raises(TypeError):
        call()


P = C.c_void_p(4096)  # never followed: every call below is refused before a launch
ODD = C.c_void_p(4098)
LIST = dict(points=P, type=0, n=10, d=8, ld=8, queries=P, nq=3, ld_q=8, scale=1.0, ids=P, m=4, offset=None, logp=P, lse=P, stream=None)
LGRAD = dict(points=P, type=0, n=10, d=8, ld=8, queries=P, nq=3, ld_q=8, scale=1.0, ids=P, m=4, logp=P, up=P, up_l=None, do=P, dq=P, ld_dq=8, dx=P, ld_dx=8, accumulate=0,
             scratch=P, bytes=1 << 40, stream=None)
DIST = dict(logp=P, teacher=P, type=0, rows=3, m=4, ld=4, lse=None, temperature=1.0, loss=P, stream=None)
DGRAD = dict(logp=P, teacher=P, type=0, rows=3, m=4, ld=4, lse=None, temperature=1.0, up=P, loss=P, out=P, stream=None)
PREF = dict(logp=P, ref=None, mask=None, tokens=9, offsets=P, pairs=1, beta=0.1, margin=0.0, smoothing=0.0, average=0, loss=P, logit=P, reward=None, scratch=P, bytes=1 << 40, stream=None)
FGRAD = dict(logp=P, ref=None, mask=None, tokens=9, offsets=P, pairs=1, beta=0.1, margin=0.0, smoothing=0.0, average=0, up=P, loss=P, logit=P, reward=None, out=P,
             scratch=P, bytes=1 << 40, stream=None)
POL = dict(logp=P, old=P, ref=None, adv=P, each=0, mask=None, tokens=9, offsets=P, sequences=2, low=0.2, high=0.2, kl=0.0, average=1, loss=P, kl_out=None, clipped=None, scratch=P,
           bytes=1 << 40, stream=None)
OGRAD = dict(logp=P, old=P, ref=None, adv=P, each=0, mask=None, tokens=9, offsets=P, sequences=2, low=0.2, high=0.2, kl=0.0, average=1, up=P, loss=P, kl_out=None, clipped=None, out=P,
             scratch=P, bytes=1 << 40, stream=None)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("name,base,change", [
    ("avq_list_log_probs", LIST, dict(points=None)), ("avq_list_log_probs", LIST, dict(queries=None)), ("avq_list_log_probs", LIST, dict(ids=None)),
    ("avq_list_log_probs", LIST, dict(logp=None)), ("avq_list_log_probs", LIST, dict(lse=None)), ("avq_list_log_probs", LIST, dict(type=3)),
    ("avq_list_log_probs", LIST, dict(n=0)), ("avq_list_log_probs", LIST, dict(n=1 << 31)), ("avq_list_log_probs", LIST, dict(d=0)), ("avq_list_log_probs", LIST, dict(ld=7)),
    ("avq_list_log_probs", LIST, dict(ld_q=7)), ("avq_list_log_probs", LIST, dict(m=-1)), ("avq_list_log_probs", LIST, dict(m=4097)), ("avq_list_log_probs", LIST, dict(nq=-1)),
    ("avq_list_log_probs", LIST, dict(nq=(1 << 19) + 1)), ("avq_list_log_probs", LIST, dict(nq=1 << 19, m=1024)), ("avq_list_log_probs", LIST, dict(scale=0.0)),
    ("avq_list_log_probs", LIST, dict(scale=NAN)), ("avq_list_log_probs", LIST, dict(points=ODD)), ("avq_list_log_probs", LIST, dict(d=16385, ld=20000, ld_q=20000)),
    ("avq_list_log_probs_grad", LGRAD, dict(logp=None)), ("avq_list_log_probs_grad", LGRAD, dict(up=None)), ("avq_list_log_probs_grad", LGRAD, dict(do=None)),
    ("avq_list_log_probs_grad", LGRAD, dict(ids=None)), ("avq_list_log_probs_grad", LGRAD, dict(ld_dq=7)), ("avq_list_log_probs_grad", LGRAD, dict(ld_dx=7)),
    ("avq_list_log_probs_grad", LGRAD, dict(dx=ODD)), ("avq_list_log_probs_grad", LGRAD, dict(m=4000, scratch=None)), ("avq_list_log_probs_grad", LGRAD, dict(m=4000, bytes=64)),
    ("avq_list_log_probs_grad", LGRAD, dict(m=4000, scratch=C.c_void_p(4100))),
    ("avq_distill_loss", DIST, dict(logp=None)), ("avq_distill_loss", DIST, dict(teacher=None)), ("avq_distill_loss", DIST, dict(loss=None)), ("avq_distill_loss", DIST, dict(ld=3)),
    ("avq_distill_loss", DIST, dict(m=4097, ld=4097)), ("avq_distill_loss", DIST, dict(m=-1)), ("avq_distill_loss", DIST, dict(rows=-1)), ("avq_distill_loss", DIST, dict(type=7)),
    ("avq_distill_loss", DIST, dict(rows=(1 << 28) + 1)), ("avq_distill_loss", DIST, dict(temperature=0.0)), ("avq_distill_loss", DIST, dict(temperature=-1.0)),
    ("avq_distill_loss", DIST, dict(temperature=NAN)), ("avq_distill_loss", DIST, dict(temperature=INF)), ("avq_distill_loss", DIST, dict(temperature=1e-310)),
    ("avq_distill_loss", DIST, dict(teacher=ODD)),
    ("avq_distill_loss_grad", DGRAD, dict(up=None)), ("avq_distill_loss_grad", DGRAD, dict(out=None)), ("avq_distill_loss_grad", DGRAD, dict(temperature=0.0)),
    ("avq_preference_loss", PREF, dict(logp=None)), ("avq_preference_loss", PREF, dict(offsets=None)), ("avq_preference_loss", PREF, dict(loss=None)),
    ("avq_preference_loss", PREF, dict(logit=None)), ("avq_preference_loss", PREF, dict(tokens=-1)), ("avq_preference_loss", PREF, dict(tokens=(1 << 28) + 1)),
    ("avq_preference_loss", PREF, dict(pairs=-1)), ("avq_preference_loss", PREF, dict(pairs=(1 << 22) + 1)), ("avq_preference_loss", PREF, dict(beta=INF)),
    ("avq_preference_loss", PREF, dict(margin=NAN)), ("avq_preference_loss", PREF, dict(smoothing=1.5)), ("avq_preference_loss", PREF, dict(smoothing=-0.1)),
    ("avq_preference_loss", PREF, dict(smoothing=NAN)),
    ("avq_preference_loss_grad", FGRAD, dict(up=None)), ("avq_preference_loss_grad", FGRAD, dict(out=None)), ("avq_preference_loss_grad", FGRAD, dict(smoothing=2.0)),
    ("avq_policy_loss", POL, dict(logp=None)), ("avq_policy_loss", POL, dict(old=None)), ("avq_policy_loss", POL, dict(adv=None)), ("avq_policy_loss", POL, dict(offsets=None)),
    ("avq_policy_loss", POL, dict(loss=None)), ("avq_policy_loss", POL, dict(kl=0.1)), ("avq_policy_loss", POL, dict(kl=-0.1)), ("avq_policy_loss", POL, dict(kl=NAN)),
    ("avq_policy_loss", POL, dict(low=-0.1)), ("avq_policy_loss", POL, dict(low=1.1)), ("avq_policy_loss", POL, dict(high=-0.1)), ("avq_policy_loss", POL, dict(high=INF)),
    ("avq_policy_loss", POL, dict(sequences=-1)), ("avq_policy_loss", POL, dict(sequences=(1 << 23) + 1)), ("avq_policy_loss", POL, dict(tokens=-5)),
    ("avq_policy_loss", POL, dict(tokens=100_000, scratch=None)), ("avq_policy_loss_grad", OGRAD, dict(tokens=100_000, bytes=8)),
    ("avq_preference_loss", PREF, dict(tokens=100_000, scratch=None)), ("avq_preference_loss_grad", FGRAD, dict(tokens=100_000, scratch=C.c_void_p(4100))),
    ("avq_policy_loss_grad", OGRAD, dict(up=None)), ("avq_policy_loss_grad", OGRAD, dict(out=None)), ("avq_policy_loss_grad", OGRAD, dict(kl=0.1)),
])
def test_c_calls_refuse(name, base, change):
    L = avq.lib()
    args = dict(base, **change)
    assert getattr(L, name)(*args.values()) == avq.AVQ_EINVAL
    assert len(L.avq_last_error()) > 0


def test_scratch_sizes():
    L = avq.lib()
    assert L.avq_list_log_probs_grad_scratch(10, 8, 0, 4) == 0
    assert L.avq_list_log_probs_grad_scratch(10, 8, 3, 0) == 0
    assert L.avq_list_log_probs_grad_scratch(10, 8, 3, 4) >= 0
    assert L.avq_list_log_probs_grad_scratch(10, 8, 3, 4000) > 0
    assert L.avq_list_log_probs_grad_scratch(10, 0, 3, 4) == avq.AVQ_EINVAL
    assert L.avq_list_log_probs_grad_scratch(10, 8, 3, 4097) == avq.AVQ_EINVAL
    assert 0 < L.avq_list_log_probs_grad_scratch(670_091, 1024, 1024, 64) < 1 << 30
    assert L.avq_preference_loss_scratch(-1, 1) == avq.AVQ_EINVAL
    assert L.avq_preference_loss_scratch(1 << 28, 1 << 22) == 0 and L.avq_preference_loss_scratch(1000, 4) == 0
    assert L.avq_policy_loss_scratch(10, -1) == avq.AVQ_EINVAL
    assert 0 < L.avq_policy_loss_scratch(1 << 28, 1) < 1 << 20
    assert 0 < L.avq_policy_loss_scratch(1 << 28, 255) < 1 << 20


def test_a_student_of_lists_alone_takes_no_lse_of_the_teacher():
    """Its list has all of its probability: the loss would have a term that no gradient moves."""
    from paper_1908_10396_amd import learn
    model = learn.Model(20, 8, device="cpu")
    with pytest.raises(ValueError, match="teacher_lse"):
        model.distill_gradients(i32(3), i32(3, 4), f32(3, 4), f32(3), listed=True)
