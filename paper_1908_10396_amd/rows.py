"""Binding of the operators on rows of learned vectors (include/avq.h): argument marshalling only.

Rows are torch tensors on the GPU of dtype float32, bfloat16 or float16, one dtype a
call; 2-D tensors may have any row stride (slices of wider matrices), with the elements of
a row side by side. Ids are int32; an id outside [0, n) is padding. Scratch and
results come from torch's allocator on the stream that the call runs on.

None of this takes part in torch's autograd: results have no history, whatever their
inputs require, and a model gets its gradients by calling the *_grad forms itself (as
`learn.Model.gradients` does).
"""
import collections
import contextlib

import torch

from . import _check, _check_shape, _dev, lib

F32, BF16, F16 = 0, 1, 2
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

LogProbs = collections.namedtuple("LogProbs", "logp lse entropy alt_ids alt_logp")
LogProbs.__doc__ = """What log_probs returns: logp (log probabilities of the given ids, None without ids), lse and entropy [nq] (fp32),
alt_ids (int32) and alt_logp [nq][k] (None for k = 0)."""

ListLogProbs = collections.namedtuple("ListLogProbs", "logp lse")
ListLogProbs.__doc__ = """What list_log_probs returns: logp [nq][m] and lse [nq] (fp32)."""


def _type(t, what):
    kind = _TYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if kind is None:
        raise TypeError("%s must be a CUDA tensor of dtype float32, bfloat16 or float16" % what)
    return kind


def _matrix(t, what, cols=None, rows=None, like=None):
    """Checks a 2-D tensor of rows. Returns (pointer, row stride)."""
    shape = t.shape
    if len(shape) != 2 or (cols is not None and shape[1] != cols) or (rows is not None and shape[0] != rows):
        raise ValueError("%s: shape %s, expected (%s, %s)" % (what, tuple(t.shape), "*" if rows is None else rows, "*" if cols is None else cols))
    if like is not None and t.dtype != like.dtype:
        raise TypeError("%s: dtype %s, expected %s" % (what, t.dtype, like.dtype))
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError("%s: the elements of a row must lie side by side" % what)
    if shape[0] <= 1:
        ld = max(shape[1], 1)
    if ld < shape[1]:
        raise ValueError("%s: rows must not overlap" % what)
    return t.data_ptr(), ld


def _vector(t, what, n, dtype):
    """Pointer of a contiguous tensor of n elements, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise TypeError("%s must be a contiguous CUDA tensor of dtype %s" % (what, dtype))
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: shape %s, expected %d contiguous elements" % (what, tuple(t.shape), n))
    return t.data_ptr()


def _ids(ids, what="ids"):
    if not isinstance(ids, torch.Tensor) or ids.dtype != torch.int32 or not ids.is_contiguous():
        raise TypeError("%s must be a contiguous CUDA tensor of dtype torch.int32" % what)
    return ids


def _same_device(first, *others):
    """All shapes and dtypes are checked before any device, as elsewhere in this package."""
    if not first.is_cuda:
        raise TypeError("tensors must be on the GPU")
    for t in others:
        if t is not None and t.device != first.device:
            raise TypeError("tensors on %s and %s" % (first.device, t.device))


@contextlib.contextmanager
def _elsewhere(device, stream):
    with torch.cuda.device(device):
        if stream is None:
            yield torch.cuda.current_stream().cuda_stream
            return
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else torch.cuda.default_stream(device)
        with torch.cuda.stream(stream):
            yield stream.cuda_stream


class _Here:
    __slots__ = ("stream",)

    def __enter__(self):
        return self.stream

    def __exit__(self, *exc):
        return False


def _on(t, stream):
    """The device of `t`, and a stream of it as torch's current one, so that what is allocated belongs to it; gives its pointer.
    (A single token's call is host time: the current stream of the current device, the usual case, changes nothing of torch's,
    which would take 5 us of a lookup's 14.)"""
    device = t.device
    if stream is not None or device.index != torch.cuda.current_device():
        return _elsewhere(device, stream)
    here = _Here()
    here.stream = torch._C._cuda_getCurrentRawStream(device.index)
    return here


def _scratch(nbytes, device):
    if nbytes < 0:
        _check(nbytes)
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def embed(table, ids, scale=1.0, out=None, stream=None):
    """avq_embed: scale * table[ids], a row of zeros for padding. ids: any shape; returns ids.shape + (d,)."""
    kind = _type(table, "table")
    tp, ld = _matrix(table, "table")
    ids = _ids(ids)
    n, d = table.shape
    if out is not None:
        if out.dtype != table.dtype:
            raise TypeError("out: dtype %s, expected %s" % (out.dtype, table.dtype))
        if tuple(out.shape) != tuple(ids.shape) + (d,) or (out.dim() != 2 and not out.is_contiguous()):
            raise ValueError("out: shape %s, expected %s, contiguous unless it has two dimensions" % (tuple(out.shape), tuple(ids.shape) + (d,)))
    _same_device(table, ids, out)
    with _on(table, stream) as st:
        if out is None:
            out = torch.empty(tuple(ids.shape) + (d,), dtype=table.dtype, device=table.device)
        op, lo = _matrix(out, "out") if out.dim() == 2 else (out.data_ptr(), d)
        _check(lib().avq_embed(tp, kind, n, d, ld, ids.data_ptr(), ids.numel(), scale, op, lo, st))
    return out


def embed_grad(grad, ids, n=None, scale=1.0, out=None, accumulate=False, stream=None):
    """avq_embed_grad: the gradient of a table of n rows from that of embed(table, ids, scale). grad: ids.shape + (d,), or
    (count, d). With `out` the result goes there, and is added to it with accumulate=True."""
    kind = _type(grad, "grad")
    ids = _ids(ids)
    if grad.dim() != 2:
        if grad.dim() == 0 or tuple(grad.shape[:-1]) != tuple(ids.shape) or not grad.is_contiguous():
            raise ValueError("grad: shape %s, expected %s + (d,), contiguous unless it has two dimensions" % (tuple(grad.shape), tuple(ids.shape)))
        d, gp, lg = grad.shape[-1], grad.data_ptr(), grad.shape[-1]
    else:
        d = grad.shape[1]
        gp, lg = _matrix(grad, "grad", rows=ids.numel())
    if out is not None:
        _type(out, "out")
        _matrix(out, "out", cols=d, rows=n, like=grad)
        n = out.shape[0]
    elif accumulate:
        raise ValueError("accumulate needs out")
    if n is None:
        raise ValueError("n or out is needed")
    _same_device(grad, ids, out)
    with _on(grad, stream) as st:
        ws = _scratch(lib().avq_embed_grad_scratch(n, d, ids.numel()), grad.device)
        if out is None:
            out = torch.empty((n, d), dtype=grad.dtype, device=grad.device)
        op, lo = _matrix(out, "out")
        _check(lib().avq_embed_grad(gp, kind, lg, ids.data_ptr(), ids.numel(), scale, op, n, d, lo, 1 if accumulate else 0,
                                     ws.data_ptr(), ws.numel(), st))
    return out


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """avq_layer_norm of the rows of a 2-D tensor. Returns (y, mean, rstd), the last two fp32 [rows], for layer_norm_grad."""
    kind = _type(x, "x")
    xp, lx = _matrix(x, "x")
    rows, d = x.shape
    wp, bp = _vector(weight, "weight", d, x.dtype), _vector(bias, "bias", d, x.dtype)
    if out is not None:
        _type(out, "out")
        _matrix(out, "out", cols=d, rows=rows, like=x)
    _same_device(x, weight, bias, out)
    with _on(x, stream) as st:
        if out is None:
            out = torch.empty((rows, d), dtype=x.dtype, device=x.device)
        stat = torch.empty((2, rows), dtype=torch.float32, device=x.device)
        mean, rstd = stat.unbind(0)
        op, lo = _matrix(out, "out")
        _check(lib().avq_layer_norm(xp, kind, rows, d, lx, wp, bp, eps, op, lo, mean.data_ptr(), rstd.data_ptr(), st))
    return out, mean, rstd


def layer_norm_grad(grad, x, mean, rstd, weight=None, out=None, stream=None):
    """avq_layer_norm_grad. Returns (dx, dweight, dbias)."""
    kind = _type(x, "x")
    _type(grad, "grad")
    xp, lx = _matrix(x, "x")
    rows, d = x.shape
    gp, lg = _matrix(grad, "grad", cols=d, rows=rows, like=x)
    mp, rp = _vector(mean, "mean", rows, torch.float32), _vector(rstd, "rstd", rows, torch.float32)
    wp = _vector(weight, "weight", d, x.dtype)
    if out is not None:
        _type(out, "out")
        _matrix(out, "out", cols=d, rows=rows, like=x)
    _same_device(x, grad, mean, rstd, weight, out)
    with _on(x, stream) as st:
        ws = _scratch(lib().avq_layer_norm_grad_scratch(rows, d), x.device)
        if out is None:
            out = torch.empty((rows, d), dtype=x.dtype, device=x.device)
        dw, db = torch.empty(d, dtype=x.dtype, device=x.device), torch.empty(d, dtype=x.dtype, device=x.device)
        op, lo = _matrix(out, "out")
        _check(lib().avq_layer_norm_grad(gp, kind, lg, xp, lx, rows, d, mp, rp, wp, op, lo, dw.data_ptr(), db.data_ptr(),
                                          ws.data_ptr(), ws.numel(), st))
    return out, dw, db


def _given(ids, nq):
    """(ids, m): ids [nq] or [nq][m], or None."""
    if ids is None:
        return None, 0
    ids = _ids(ids)
    if ids.dim() not in (1, 2) or ids.shape[0] != nq:
        raise ValueError("ids: shape %s, expected (%d,) or (%d, *)" % (tuple(ids.shape), nq, nq))
    return ids, 1 if ids.dim() == 1 else ids.shape[1]


def _prob_outputs(ids, nq, k, device):
    f32 = dict(dtype=torch.float32, device=device)
    logp = None if ids is None else torch.empty(tuple(ids.shape), **f32)
    stat = torch.empty((2, nq), **f32)
    alt = (torch.empty((nq, k), dtype=torch.int32, device=device), torch.empty((nq, k), **f32)) if k else (None, None)
    return LogProbs(logp, *stat.unbind(0), *alt)


def _ptr(t):
    return None if t is None else t.data_ptr()


def log_probs(points, queries, ids=None, k=0, scale=1.0, stream=None):
    """avq_log_probs: the softmax over all rows of `points` of scale * <query, row>. ids: [nq] or [nq][m], whose log
    probabilities are wanted; k: how many of the best rows. Returns LogProbs."""
    kind = _type(points, "points")
    _type(queries, "queries")
    pp, lp = _matrix(points, "points")
    n, d = points.shape
    qp, lq = _matrix(queries, "queries", cols=d, like=points)
    nq, k = queries.shape[0], int(k)
    ids, m = _given(ids, nq)
    _same_device(points, queries, ids)
    with _on(points, stream) as st:
        ws = _scratch(lib().avq_log_probs_scratch(kind, n, d, nq, m, k), points.device)
        r = _prob_outputs(ids, nq, k, points.device)
        _check(lib().avq_log_probs(pp, kind, n, d, lp, qp, nq, lq, scale, _ptr(ids), m, _ptr(r.logp), _ptr(r.lse), _ptr(r.entropy), k,
                                    _ptr(r.alt_ids), _ptr(r.alt_logp), ws.data_ptr(), ws.numel(), st))
    return r


def _index_log_probs(index, queries, ids, k, scale, stream):
    _check_shape(queries, (None, index.d), "queries")
    nq, k = queries.shape[0], int(k)
    ids, m = _given(ids, nq)
    if not 0 <= k <= 512:
        raise ValueError("k must be 0 .. 512, got %d" % k)
    qp = _dev(queries, torch.float32, "queries", (None, index.d))
    _same_device(queries, ids)
    with _on(queries, stream) as st:
        r = _prob_outputs(ids, nq, k, queries.device)
        _check(lib().avq_index_log_probs(index._h, qp, nq, scale, _ptr(ids), m, _ptr(r.logp), _ptr(r.lse), _ptr(r.entropy), k,
                                          _ptr(r.alt_ids), _ptr(r.alt_logp), st))
    return r


def log_probs_grad(points, queries, ids, lse, grad_logp, entropy=None, grad_entropy=None, grad_lse=None, scale=1.0,
                   out_points=None, accumulate=False, stream=None):
    """avq_log_probs_grad: (dqueries, dpoints) for the gradients of the loss with respect to the results of
    log_probs(points, queries, ids, scale=scale): grad_logp (shaped like ids; None with ids=None), grad_entropy and
    grad_lse [nq] or None. lse, and entropy where it has a gradient, are that call's. With out_points dpoints goes there,
    and is added to it with accumulate=True."""
    kind = _type(points, "points")
    _type(queries, "queries")
    pp, lp = _matrix(points, "points")
    n, d = points.shape
    qp, lq = _matrix(queries, "queries", cols=d, like=points)
    nq = queries.shape[0]
    ids, m = _given(ids, nq)
    if (ids is None) != (grad_logp is None):
        raise ValueError("ids and grad_logp come together")
    f32 = torch.float32
    up = _vector(grad_logp, "grad_logp", nq * m, f32)
    lsep, entp = _vector(lse, "lse", nq, f32), _vector(entropy, "entropy", nq, f32)
    upe, upl = _vector(grad_entropy, "grad_entropy", nq, f32), _vector(grad_lse, "grad_lse", nq, f32)
    if out_points is not None:
        _type(out_points, "out_points")
        _matrix(out_points, "out_points", cols=d, rows=n, like=points)
    elif accumulate:
        raise ValueError("accumulate needs out_points")
    _same_device(points, queries, ids, lse, grad_logp, entropy, grad_entropy, grad_lse, out_points)
    with _on(points, stream) as st:
        ws = _scratch(lib().avq_log_probs_grad_scratch(kind, n, d, nq, m), points.device)
        dq = torch.empty((nq, d), dtype=points.dtype, device=points.device)
        if out_points is None:
            out_points = torch.empty((n, d), dtype=points.dtype, device=points.device)
        op, lo = _matrix(out_points, "out_points")
        _check(lib().avq_log_probs_grad(pp, kind, n, d, lp, qp, nq, lq, scale, _ptr(ids), m, lsep, entp, up, upe, upl, dq.data_ptr(), d,
                                         op, lo, 1 if accumulate else 0, ws.data_ptr(), ws.numel(), st))
    return dq, out_points


def _listed(ids, nq):
    ids = _ids(ids)
    if ids.dim() != 2 or ids.shape[0] != nq:
        raise ValueError("ids: shape %s, expected (%d, *)" % (tuple(ids.shape), nq))
    return ids, ids.shape[1]


def list_log_probs(points, queries, ids, offset=None, scale=1.0, stream=None):
    """avq_list_log_probs: the softmax over each query's own list of rows, ids [nq][m], of scale * <query, row> + offset
    (fp32 [nq][m] or None). Returns ListLogProbs."""
    kind = _type(points, "points")
    _type(queries, "queries")
    pp, lp = _matrix(points, "points")
    n, d = points.shape
    qp, lq = _matrix(queries, "queries", cols=d, like=points)
    nq = queries.shape[0]
    ids, m = _listed(ids, nq)
    op = _vector(offset, "offset", nq * m, torch.float32)
    _same_device(points, queries, ids, offset)
    with _on(points, stream) as st:
        logp = torch.empty((nq, m), dtype=torch.float32, device=points.device)
        lse = torch.empty(nq, dtype=torch.float32, device=points.device)
        _check(lib().avq_list_log_probs(pp, kind, n, d, lp, qp, nq, lq, scale, ids.data_ptr(), m, op, logp.data_ptr(), lse.data_ptr(), st))
    return ListLogProbs(logp, lse)


def list_log_probs_grad(points, queries, ids, logp, grad_logp, grad_lse=None, scale=1.0, out_points=None, accumulate=False, stream=None):
    """avq_list_log_probs_grad: (dqueries, dpoints, doffset) for the gradients of the loss with respect to the results of
    list_log_probs(points, queries, ids, scale=scale), grad_logp [nq][m] and grad_lse [nq] or None; logp is that call's.
    With out_points dpoints goes there, and is added to it with accumulate=True."""
    kind = _type(points, "points")
    _type(queries, "queries")
    pp, lp = _matrix(points, "points")
    n, d = points.shape
    qp, lq = _matrix(queries, "queries", cols=d, like=points)
    nq = queries.shape[0]
    ids, m = _listed(ids, nq)
    f32 = torch.float32
    logpp, up, upl = _vector(logp, "logp", nq * m, f32), _vector(grad_logp, "grad_logp", nq * m, f32), _vector(grad_lse, "grad_lse", nq, f32)
    if logp is None or grad_logp is None:
        raise ValueError("logp and grad_logp are needed")
    if out_points is not None:
        _type(out_points, "out_points")
        _matrix(out_points, "out_points", cols=d, rows=n, like=points)
    elif accumulate:
        raise ValueError("accumulate needs out_points")
    _same_device(points, queries, ids, logp, grad_logp, grad_lse, out_points)
    with _on(points, stream) as st:
        need = lib().avq_list_log_probs_grad_scratch(n, d, nq, m)
        ws = None if need == 0 else _scratch(need, points.device)
        dq = torch.empty((nq, d), dtype=points.dtype, device=points.device)
        do = torch.empty((nq, m), dtype=f32, device=points.device)
        if out_points is None:
            out_points = torch.empty((n, d), dtype=points.dtype, device=points.device)
        op, lo = _matrix(out_points, "out_points")
        _check(lib().avq_list_log_probs_grad(pp, kind, n, d, lp, qp, nq, lq, scale, ids.data_ptr(), m, logpp, up, upl, do.data_ptr(), dq.data_ptr(), d,
                                              op, lo, 1 if accumulate else 0, _ptr(ws), 0 if ws is None else ws.numel(), st))
    return dq, out_points, do
