"""What the operators on rows refuse, before any pointer reaches the GPU."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")


def f32(*shape):
    return torch.zeros(shape)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: avq.embed(f32(4), i32(2)),                                       # a table has two dimensions
    lambda: avq.embed(f32(4, 8).t(), i32(2)),                                # elements of a row side by side
    lambda: avq.embed(f32(1, 8).expand(4, 8), i32(2)),                       # rows over one another
    lambda: avq.embed(f32(4, 8), i32(2), out=f32(3, 8)),
    lambda: avq.embed_grad(f32(3, 8), i32(2), 10),
    lambda: avq.embed_grad(f32(2, 8), i32(2)),                               # neither n nor out
    lambda: avq.embed_grad(f32(2, 8), i32(2), 10, accumulate=True),
    lambda: avq.embed_grad(f32(2, 8), i32(2), 10, out=f32(9, 8)),
    lambda: avq.layer_norm(f32(3, 8), f32(7)),
    lambda: avq.layer_norm(f32(3, 8), out=f32(3, 9)),
    lambda: avq.layer_norm_grad(f32(3, 8), f32(3, 9), f32(3), f32(3)),
    lambda: avq.layer_norm_grad(f32(3, 8), f32(3, 8), f32(2), f32(3)),
    lambda: avq.log_probs(f32(10, 8), f32(3, 9)),
    lambda: avq.log_probs(f32(10, 8), f32(3, 8), i32(4)),
    lambda: avq.log_probs(f32(10, 8), f32(3, 8), i32(3, 1, 1)),
    lambda: avq.log_probs_grad(f32(10, 8), f32(3, 8), i32(3), f32(3), None),
    lambda: avq.log_probs_grad(f32(10, 8), f32(3, 8), i32(3), f32(3), f32(4)),
    lambda: avq.log_probs_grad(f32(10, 8), f32(3, 8), i32(3), f32(2), f32(3)),
    lambda: avq.log_probs_grad(f32(10, 8), f32(3, 8), i32(3), f32(3), f32(3), accumulate=True),
    lambda: avq.log_probs_grad(f32(10, 8), f32(3, 8), i32(3), f32(3), f32(3), out_points=f32(9, 8)),
])
def test_shapes(call):
    with pytest.raises(ValueError):
        call()


@pytest.mark.parametrize("call", [
    lambda: avq.embed(f32(4, 8).double(), i32(2)),
    lambda: avq.embed(f32(4, 8), i32(2).long()),
    lambda: avq.embed(f32(4, 8), i32(4)[::2]),
    lambda: avq.embed(f32(4, 8), i32(2), out=f32(2, 8).half()),
    lambda: avq.embed_grad(f32(2, 8), i32(2), out=f32(9, 8).half()),
    lambda: avq.layer_norm(f32(3, 8), f32(8).half()),
    lambda: avq.layer_norm_grad(f32(3, 8).half(), f32(3, 8), f32(3), f32(3)),
    lambda: avq.layer_norm_grad(f32(3, 8), f32(3, 8), f32(3).double(), f32(3)),
    lambda: avq.log_probs(f32(10, 8), f32(3, 8).bfloat16()),
    lambda: avq.log_probs(f32(10, 8), f32(3, 8), i32(3).long()),
    lambda: avq.log_probs_grad(f32(10, 8), f32(3, 8), i32(3), f32(3), f32(3).half()),
    # right shapes and types, but on the host
    lambda: avq.embed(f32(4, 8), i32(2)),
    lambda: avq.embed_grad(f32(2, 8), i32(2), 4),
    lambda: avq.layer_norm(f32(3, 8)),
    lambda: avq.log_probs(f32(10, 8), f32(3, 8)),
])
def test_types_and_devices(call):
    with pytest.raises(TypeError):
        call()


P = C.c_void_p(4096)  # never followed: every call below is refused before a launch
EMBED = dict(table=P, type=0, n=10, d=8, ld=8, ids=P, count=3, scale=1.0, out=P, ld_out=8, stream=None)
GRAD = dict(grad=P, type=0, ld=8, ids=P, count=3, scale=1.0, out=P, n=10, d=8, ld_out=8, accumulate=0, scratch=P, bytes=1 << 30, stream=None)
NORM = dict(x=P, type=0, rows=3, d=8, ld=8, weight=None, bias=None, eps=1e-5, y=P, ld_y=8, mean=None, rstd=None, stream=None)
NGRAD = dict(grad=P, type=0, ld=8, x=P, ld_x=8, rows=3, d=8, mean=P, rstd=P, weight=None, dx=P, ld_dx=8, dw=None, db=None, scratch=P, bytes=1 << 30, stream=None)
PROBS = dict(points=P, type=0, n=10, d=8, ld=8, queries=P, nq=3, ld_q=8, scale=1.0, ids=None, m=0, logp=None, lse=P, entropy=None, k=0, alt=None, altp=None,
             scratch=P, bytes=1 << 40, stream=None)
PGRAD = dict(points=P, type=0, n=10, d=8, ld=8, queries=P, nq=3, ld_q=8, scale=1.0, ids=P, m=1, lse=P, entropy=None, up=P, up_h=None, up_l=None, dq=P, ld_dq=8,
             dx=P, ld_dx=8, accumulate=0, scratch=P, bytes=1 << 40, stream=None)
ODD = C.c_void_p(4098)


@pytest.mark.parametrize("name,base,change", [
    ("avq_embed", EMBED, dict(table=None)), ("avq_embed", EMBED, dict(out=None)), ("avq_embed", EMBED, dict(ids=None)),
    ("avq_embed", EMBED, dict(type=3)), ("avq_embed", EMBED, dict(n=0)), ("avq_embed", EMBED, dict(n=1 << 31)), ("avq_embed", EMBED, dict(d=0)),
    ("avq_embed", EMBED, dict(d=16385, ld=20000, ld_out=20000)), ("avq_embed", EMBED, dict(ld=7)), ("avq_embed", EMBED, dict(ld_out=7)),
    ("avq_embed", EMBED, dict(count=-1)), ("avq_embed", EMBED, dict(count=(1 << 28) + 1)), ("avq_embed", EMBED, dict(table=ODD)),
    ("avq_embed_grad", GRAD, dict(grad=None)), ("avq_embed_grad", GRAD, dict(ids=None)), ("avq_embed_grad", GRAD, dict(out=None)),
    ("avq_embed_grad", GRAD, dict(scratch=None)), ("avq_embed_grad", GRAD, dict(bytes=100)), ("avq_embed_grad", GRAD, dict(scratch=C.c_void_p(4100))),
    ("avq_embed_grad", GRAD, dict(ld=1)), ("avq_embed_grad", GRAD, dict(type=-1)),
    ("avq_layer_norm", NORM, dict(x=None)), ("avq_layer_norm", NORM, dict(y=None)), ("avq_layer_norm", NORM, dict(eps=-1.0)),
    ("avq_layer_norm", NORM, dict(eps=float("nan"))), ("avq_layer_norm", NORM, dict(rows=-1)), ("avq_layer_norm", NORM, dict(ld_y=2)),
    ("avq_layer_norm", NORM, dict(weight=ODD)),
    ("avq_layer_norm_grad", NGRAD, dict(mean=None)), ("avq_layer_norm_grad", NGRAD, dict(dx=None)), ("avq_layer_norm_grad", NGRAD, dict(bytes=8)),
    ("avq_layer_norm_grad", NGRAD, dict(db=ODD)),
    ("avq_log_probs", PROBS, dict(points=None)), ("avq_log_probs", PROBS, dict(queries=None)), ("avq_log_probs", PROBS, dict(lse=None)),
    ("avq_log_probs", PROBS, dict(scale=0.0)), ("avq_log_probs", PROBS, dict(scale=float("inf"))), ("avq_log_probs", PROBS, dict(scale=float("nan"))),
    ("avq_log_probs", PROBS, dict(k=11, alt=P, altp=P)), ("avq_log_probs", PROBS, dict(n=1000, k=513, alt=P, altp=P)), ("avq_log_probs", PROBS, dict(k=1)),
    ("avq_log_probs", PROBS, dict(m=1)), ("avq_log_probs", PROBS, dict(m=-1)), ("avq_log_probs", PROBS, dict(m=4097, ids=P, logp=P)),
    ("avq_log_probs", PROBS, dict(nq=-1)), ("avq_log_probs", PROBS, dict(nq=(1 << 19) + 1)), ("avq_log_probs", PROBS, dict(bytes=1)),
    ("avq_log_probs", PROBS, dict(n=1000, d=16384, ld=16384, ld_q=16384, k=512, alt=P, altp=P)),
    ("avq_log_probs_grad", PGRAD, dict(lse=None)), ("avq_log_probs_grad", PGRAD, dict(up=None)), ("avq_log_probs_grad", PGRAD, dict(ids=None)),
    ("avq_log_probs_grad", PGRAD, dict(up_h=P)), ("avq_log_probs_grad", PGRAD, dict(ld_dx=3)), ("avq_log_probs_grad", PGRAD, dict(scale=0.0)),
    ("avq_log_probs_grad", PGRAD, dict(scratch=None)), ("avq_log_probs_grad", PGRAD, dict(dq=ODD)),
])
def test_c_calls_refuse(name, base, change):
    L = avq.lib()
    args = dict(base, **change)
    assert getattr(L, name)(*args.values()) == avq.AVQ_EINVAL
    assert len(L.avq_last_error()) > 0


def test_scratch_sizes():
    L = avq.lib()
    assert L.avq_embed_grad_scratch(10, 8, 0) == 0
    assert L.avq_embed_grad_scratch(10, 8, 5) > 0
    assert L.avq_embed_grad_scratch(0, 8, 5) == avq.AVQ_EINVAL
    assert L.avq_layer_norm_grad_scratch(10, 0) == avq.AVQ_EINVAL
    assert L.avq_log_probs_scratch(0, 10, 8, 3, 1, 11) == avq.AVQ_EINVAL
    assert L.avq_log_probs_scratch(0, 10, 8, 0, 1, 2) == 0
    assert L.avq_log_probs_grad_scratch(9, 10, 8, 3, 1) == avq.AVQ_EINVAL
    # grows with what is asked for, and stays within a card
    assert L.avq_log_probs_scratch(0, 1_183_514, 100, 2048, 3, 10) < 1 << 32
    assert 0 < L.avq_log_probs_grad_scratch(1, 670_091, 1024, 1024, 1) < 1 << 34


def test_index_call_without_an_index():
    assert avq.lib().avq_index_log_probs(None, P, 1, 1.0, None, 0, None, P, None, 0, None, None, None) == avq.AVQ_EINVAL
