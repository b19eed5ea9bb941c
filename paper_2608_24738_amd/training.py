"""The operators of a training step on distances, over torch tensors.

``label_log_probs``  log-probabilities of given labels, with the entropy, the
                     likeliest classes and the expected value of a field under
                     the softmax (the boundary loss, for the signed distance
                     field of each class)
``relative_bias``    a learned bias by buckets of the distance between a
                     query's and a key's position
``distance_bias``    the same bias from a distance field

All three run in the HIP kernels of ``libtm_edt.so`` (``include/tm_train.h``)
on the current stream, take part in autograd (in reverse mode, once), and raise
where the library refuses a request; there is no fallback.

Small calls are bound by the host.  On one GPU a backward pass inside ``with
torch.autograd.set_multithreading_enabled(False):`` stays on the caller's
thread, which takes a forward and backward pass from some 95 to 40 us.
"""
from __future__ import annotations

import ctypes
import functools
import math
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from .binding import METRICS, _call, _sampling_array, _shape_array, load

FLOATS = {torch.float16: 4, torch.bfloat16: 5, torch.float32: 6}
LABELS = {torch.uint8: 0, torch.int32: 2, torch.int64: 3}
DISTANCES = {torch.int32: 2, torch.float32: 6}
DISTANCE_TYPES = {code: kind for kind, code in DISTANCES.items()}
BIAS_METRICS = dict(METRICS, offset=3)
MAX_TOP = 32
MAX_RECOMPUTE = 32           # classes whose gradient needs no saved statistics
MAX_BUCKETS = 256


class LabelLogProbs(NamedTuple):
    """What ``label_log_probs`` gives; None for what was not asked for."""
    log_probs: Optional[torch.Tensor]
    entropy: Optional[torch.Tensor]
    field_mean: Optional[torch.Tensor]
    top_log_probs: Optional[torch.Tensor]
    top_indices: Optional[torch.Tensor]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _collapse(sizes, strides):
    """One axis (extent, stride) that visits the elements of these axes in
    order, or None where no single stride does."""
    extent, step = 1, 0
    for n, st in zip(reversed(sizes), reversed(strides)):
        if n == 1:
            continue
        if extent == 1:
            step = st
        elif st != extent * step:
            return None
        extent *= n
    return extent, step


@functools.lru_cache(maxsize=1024)
def _view(shape, strides, dim):
    """((outer, classes, inner), their strides as a C array) of a tensor whose
    class axis is ``dim``, or None where three strides cannot describe it."""
    if 0 in shape:
        return (math.prod(shape[:dim]), shape[dim], math.prod(shape[dim + 1:])), (ctypes.c_int64 * 3)(0, 0, 0)
    outer = _collapse(shape[:dim], strides[:dim])
    inner = _collapse(shape[dim + 1:], strides[dim + 1:])
    if outer is None or inner is None:
        return None
    return (outer[0], shape[dim], inner[0]), (ctypes.c_int64 * 3)(outer[1], strides[dim], inner[1])


def _viewed(t, dim):
    """(tensor, extents, strides): ``t``, or a contiguous copy of it where its
    strides are too many."""
    view = _view(tuple(t.shape), t.stride(), dim)
    if view is None:
        t = t.contiguous()
        view = _view(tuple(t.shape), t.stride(), dim)
    return t, view[0], view[1]


@functools.lru_cache(maxsize=1024)
def _label_plan(shape, strides, dim, dtype, top_k):
    """What a forward call needs to know of logits of this shape: (extents,
    strides, shape of a value per element, shape of the top classes, bytes of
    workspace), or None where three strides cannot describe them."""
    view = _view(shape, strides, dim)
    if view is None:
        return None
    extents, steps = view
    nbytes = 0
    if extents[1] > MAX_RECOMPUTE:               # rows may be cut into parts
        nbytes = int(load().tm_label_logp_workspace_size(dtype, *extents, steps, top_k))
    return extents, steps, shape[:dim] + shape[dim + 1:], shape[:dim] + (top_k,) + shape[dim + 1:], nbytes


def _label_forward(logits, labels, field, dim, entropy, top_k, stats):
    """Runs tm_label_logp; returns (logits, field) as they were read, the outputs,
    the statistics for the gradient and what the tensors are: (axis, type, device
    and shape of the logits, type of the labels, both types' codes)."""
    dev, kind, whole = logits.device, logits.dtype, tuple(logits.shape)
    dtype = FLOATS[kind]
    plan = _label_plan(whole, logits.stride(), dim, dtype, top_k)
    if plan is None:
        logits = logits.contiguous()
        plan = _label_plan(whole, logits.stride(), dim, dtype, top_k)
    extents, strides, shape, shape_k, nbytes = plan
    field_strides = None
    if field is not None:
        field, _, field_strides = _viewed(field, dim)
    empty, f32 = torch.empty, torch.float32
    logp = empty(shape, dtype=f32, device=dev) if labels is not None else None
    ent = empty(shape, dtype=f32, device=dev) if entropy else None
    mean = empty(shape, dtype=f32, device=dev) if field is not None else None
    top = empty(shape_k, dtype=f32, device=dev) if top_k else None
    index = empty(shape_k, dtype=torch.int32, device=dev) if top_k else None
    kept = empty(shape + (2,), dtype=f32, device=dev) if stats else None
    workspace = empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    label_kind, label_dtype = (labels.dtype, LABELS[labels.dtype]) if labels is not None else (None, 0)
    _call("tm_label_logp", dev, None, logits.data_ptr(), dtype, *extents, strides, _ptr(labels), label_dtype,
          _ptr(field), field_strides, top_k, _ptr(logp), _ptr(ent), _ptr(mean), _ptr(top), _ptr(index), _ptr(kept),
          _ptr(workspace), nbytes)
    what = (dim, kind, dev, whole, label_kind, dtype, label_dtype)
    return logits, field, (logp, ent, mean, top, index), kept, what


def _upstream(grad):
    if grad is None or (grad.dtype == torch.float32 and grad.is_contiguous()):
        return grad
    return grad.to(torch.float32).contiguous()


def _restored(t, dtype, device, shape):
    """A dense tensor that autograd kept.  Hooks on saved tensors (such as
    torch.autograd.graph.save_on_cpu) may give it another layout, nothing else."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device or t.shape != shape:
        _changed()
    return t.contiguous()


def _changed():
    raise RuntimeError("a hook on saved tensors gave back another type, shape or device")


def _once():
    if torch.is_grad_enabled():
        raise RuntimeError("the training operators can be differentiated once only")


def _reverse_only(*tensors):
    """Refuses tensors with a forward-mode tangent, which the call would drop.
    (None can have one outside forward_ad.dual_level; asking each takes 0.3 us.)"""
    if forward_ad._current_level >= 0 and any(
            t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise RuntimeError("the training operators have no forward-mode derivatives")


class _LabelLogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, labels, field, dim, entropy, top_k):
        stats = logits.shape[dim] > MAX_RECOMPUTE
        logits, field, out, kept, ctx.what = _label_forward(logits, labels, field, dim, entropy, top_k, stats)
        ctx.set_materialize_grads(False)
        if top_k:
            ctx.mark_non_differentiable(out[3], out[4])
        ctx.save_for_backward(logits, labels, field, kept, out[1] if stats else None, out[2] if stats else None)
        return out

    @staticmethod
    def backward(ctx, up_logp, up_entropy, up_mean, _top, _index):
        _once()
        if up_logp is None and up_entropy is None and up_mean is None:
            return None, None, None, None, None, None
        logits, labels, field, kept, entropy, mean = ctx.saved_tensors
        dim, kind, dev, shape, label_kind, dtype, label_dtype = ctx.what
        if logits.dtype is not kind or logits.device != dev or logits.shape != shape:
            _changed()
        # strides are those of the tensors at hand, not the forward call's
        plan = _label_plan(shape, logits.stride(), dim, dtype, 0)
        if plan is None:
            logits = logits.contiguous()
            plan = _label_plan(shape, logits.stride(), dim, dtype, 0)
        extents, strides, rest = plan[:3]
        f32, field_strides = torch.float32, None
        labels = _restored(labels, label_kind, dev, rest)
        if field is not None:
            if field.dtype is not f32 or field.device != dev or field.shape != shape:
                _changed()
            view = _view(shape, field.stride(), dim)
            if view is None:
                field = field.contiguous()
                view = _view(shape, field.stride(), dim)
            field_strides = view[1]
        if kept is not None:
            kept = _restored(kept, f32, dev, rest + (2,))
            entropy, mean = _restored(entropy, f32, dev, rest), _restored(mean, f32, dev, rest)
        up_logp, up_entropy, up_mean = _upstream(up_logp), _upstream(up_entropy), _upstream(up_mean)
        grad = torch.empty_like(logits)
        grad_strides = strides
        if grad.stride() != logits.stride():
            grad, _, grad_strides = _viewed(grad, dim)
        _call("tm_label_logp_grad", dev, None, logits.data_ptr(), dtype, *extents, strides,
              _ptr(labels), label_dtype, _ptr(field), field_strides, _ptr(kept), _ptr(entropy), _ptr(mean),
              _ptr(up_logp), _ptr(up_entropy), _ptr(up_mean), grad.data_ptr(), grad_strides)
        return grad, None, None, None, None, None


def label_log_probs(logits: torch.Tensor, labels: Optional[torch.Tensor] = None, *, dim: int = 1,
                    entropy: bool = False, top_k: int = 0, field: Optional[torch.Tensor] = None) -> LabelLogProbs:
    """Log-probabilities of given labels under the softmax of ``logits`` over
    axis ``dim``: (B, C, *spatial) maps, or rows (N, C).

    ``logits``  float32, float16 or bfloat16, any strides.
    ``labels``  their shape without ``dim``; uint8, bool, int32 or int64.  A
                label outside [0, C) marks an element without one: log-probability
                0, and no gradient through it.  None: no ``log_probs``.
    ``entropy`` also the entropy of each element's classes.
    ``top_k``   also the largest log-probabilities and their classes (at most
                32), along ``dim`` in falling order, equal logits by rising class.
    ``field``   float32, the logits' shape (or broadcastable to it): also
                ``field_mean``, the sum over classes of probability x field.

    Results are float32 (indices int32).  Gradients flow to ``logits`` from
    ``log_probs``, ``entropy`` and ``field_mean``; labels, field and the top
    classes are constants of the step.
    """
    if not logits.is_cuda:
        raise ValueError("logits must be a ROCm (cuda) tensor")
    if logits.dtype not in FLOATS:
        raise TypeError("logits must be float32, float16 or bfloat16, got %s" % logits.dtype)
    if not -logits.dim() <= dim < logits.dim():
        raise ValueError("logits of %d dimensions have no axis %d" % (logits.dim(), dim))
    dim %= logits.dim()
    classes = logits.shape[dim]
    if classes < 1:
        raise ValueError("logits have no classes along axis %d" % dim)
    if labels is not None:
        if labels.device != logits.device:
            raise ValueError("labels are on %s, the logits on %s" % (labels.device, logits.device))
        if labels.dtype == torch.bool:
            labels = labels.contiguous().view(torch.uint8)
        if labels.dtype not in LABELS:
            raise TypeError("labels must be uint8, bool, int32 or int64, got %s" % labels.dtype)
        if labels.shape != logits.shape[:dim] + logits.shape[dim + 1:]:
            raise ValueError("labels of shape %s do not fit logits of shape %s with classes along axis %d"
                             % (tuple(labels.shape), tuple(logits.shape), dim))
        labels = labels.contiguous()
    if not 0 <= top_k <= min(classes, MAX_TOP):
        raise ValueError("top_k must be between 0 and %d, got %d" % (min(classes, MAX_TOP), top_k))
    if field is not None:
        if field.device != logits.device:
            raise ValueError("field is on %s, the logits on %s" % (field.device, logits.device))
        if field.dtype != torch.float32:
            raise TypeError("field must be float32, got %s" % field.dtype)
        if field.requires_grad and torch.is_grad_enabled():
            raise ValueError("field is a constant of the step; detach it")
        if field.shape != logits.shape:
            field = field.expand(logits.shape)
    if labels is None and field is None and not entropy and not top_k:
        raise ValueError("nothing to compute: give labels or a field, or ask for the entropy or top_k")
    _reverse_only(logits, field)
    entropy, top_k = bool(entropy), int(top_k)
    if logits.requires_grad and torch.is_grad_enabled():
        return LabelLogProbs(*_LabelLogProbs.apply(logits, labels, field, dim, entropy, top_k))
    return LabelLogProbs(*_label_forward(logits, labels, field, dim, entropy, top_k, False)[2])


def distance_edges(buckets: int, reach: float, *, signed: bool = False, device=None) -> torch.Tensor:
    """``buckets`` - 1 ascending edges for ``relative_bias`` and ``distance_bias``:
    one bucket a unit for the nearer half, then buckets growing by a constant
    factor up to ``reach``; ``signed`` splits them between both signs (of
    metric "offset").  Any other ascending edges do as well."""
    if not 1 <= buckets <= MAX_BUCKETS:
        raise ValueError("buckets must be between 1 and %d, got %d" % (MAX_BUCKETS, buckets))

    def half(count):
        exact = (count + 1) // 2
        far = count - exact
        span = max(float(reach), 2.0 * exact)
        return [0.5 + i for i in range(exact)] + [
            0.5 + exact * (span / max(exact, 1)) ** ((i + 1) / (far + 1)) for i in range(far)]
    if signed:
        near = half((buckets - 1) // 2)
        edges = [-e for e in reversed(near)] + near
        if len(edges) < buckets - 1:
            edges.append(2.0 * near[-1] if near else 0.5)
    else:
        edges = half(buckets - 1)
    return torch.tensor(edges, dtype=torch.float32, device=device)


class _Bias(torch.autograd.Function):
    """A bias whose table learns.  ``source`` is what the entry points take
    before the table: ("tm_distance_bias", args, keep) with ``keep`` the
    distances, or ("tm_relative_bias", args, None)."""

    @staticmethod
    def forward(ctx, table, edges, add, source, shape):
        name, args, distances = source
        ctx.save_for_backward(edges, distances)
        ctx.kind = (name + "_grad", args, table.dtype, tuple(table.shape), add is not None,
                    None if distances is None else distances.shape)
        return _bias_forward(table, edges, add, source, shape)

    @staticmethod
    def backward(ctx, up):
        _once()
        grad = None
        name, args, dtype, shape, has_add, field_shape = ctx.kind
        wanted = ctx.needs_input_grad
        if wanted[0]:
            edges, distances = ctx.saved_tensors
            up = up.contiguous()
            buckets, heads = shape
            dev = up.device
            edges = _restored(edges, torch.float32, dev, (buckets - 1,))
            grad = torch.empty(shape, dtype=dtype, device=dev)
            nbytes = _bias_workspace(buckets, heads)
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
            if distances is not None:
                distances = _restored(distances, DISTANCE_TYPES[args[1]], dev, field_shape)
                args = (distances.data_ptr(),) + args[1:]
            _call(name, dev, None, *args, up.data_ptr(), FLOATS[up.dtype], buckets, heads, edges.data_ptr(),
                  grad.data_ptr(), FLOATS[dtype], _ptr(workspace), nbytes)
        return grad, None, up if has_add and wanted[2] else None, None, None


@functools.lru_cache(maxsize=1024)
def _bias_workspace(buckets, heads):
    return int(load().tm_bias_grad_workspace_size(buckets, heads))


def _bias_forward(table, edges, add, source, shape):
    name, args, _ = source
    out = torch.empty(shape, dtype=table.dtype if add is None else add.dtype, device=table.device)
    _call(name, table.device, None, *args, table.data_ptr(), FLOATS[table.dtype], table.shape[0], table.shape[1],
          edges.data_ptr(), _ptr(add), out.data_ptr(), FLOATS[out.dtype])
    return out


def _run_bias(table, edges, add, source, shape):
    if torch.is_grad_enabled() and (table.requires_grad or (add is not None and add.requires_grad)):
        return _Bias.apply(table, edges, add, source, shape)
    return _bias_forward(table, edges, add, source, shape)


def _check_bias(table, edges, add):
    if not table.is_cuda:
        raise ValueError("table must be a ROCm (cuda) tensor")
    if table.dtype not in FLOATS:
        raise TypeError("table must be float32, float16 or bfloat16, got %s" % table.dtype)
    shape, device = table.shape, table.device
    if len(shape) != 2 or not 1 <= shape[0] <= MAX_BUCKETS or shape[1] < 1:
        raise ValueError("table must be (buckets, heads) with 1 to %d buckets, got %s" % (MAX_BUCKETS, tuple(shape)))
    if edges.dtype != torch.float32 or edges.device != device:
        raise TypeError("edges must be float32 on %s" % device)
    if edges.dim() != 1 or edges.shape[0] != shape[0] - 1:
        raise ValueError("a table of %d buckets needs %d edges, got %s" % (shape[0], shape[0] - 1, tuple(edges.shape)))
    if add is not None:
        if add.dtype not in FLOATS:
            raise TypeError("add must be float32, float16 or bfloat16, got %s" % add.dtype)
        if add.device != device:
            raise ValueError("add is on %s, the table on %s" % (add.device, device))
        add = add.contiguous()
    _reverse_only(table, edges, add)
    return table.contiguous(), edges.contiguous(), add


def distance_bias(distances: torch.Tensor, table: torch.Tensor, edges: torch.Tensor, *,
                  add: Optional[torch.Tensor] = None) -> torch.Tensor:
    """A learned bias by buckets of a distance field: from ``distances`` (B,
    *spatial), float32 or int32, to (B, heads, *spatial) with

        out[b, h, x] = table[number of edges <= distances[b, x], h]  (+ add[b, h, x])

    ``table``  (buckets, heads) float32, float16 or bfloat16.
    ``edges``  buckets - 1 ascending float32 values on the same device.
    ``add``    (B, heads, *spatial), such as logits: the sum is made in float32
               and rounded once to its type; alone, the bias has the table's.

    Gradients flow to ``table`` and ``add``; distances are constants of the step.
    """
    table, edges, add = _check_bias(table, edges, add)
    if distances.dtype not in DISTANCES:
        raise TypeError("distances must be float32 or int32, got %s" % distances.dtype)
    if distances.device != table.device:
        raise ValueError("distances are on %s, the table on %s" % (distances.device, table.device))
    if distances.dim() < 1:
        raise ValueError("distances must be (B, *spatial)")
    if distances.requires_grad and torch.is_grad_enabled():
        raise ValueError("distances are constants of the step; detach them")
    _reverse_only(distances)
    distances = distances.contiguous()
    shape = (distances.shape[0], table.shape[1]) + tuple(distances.shape[1:])
    if add is not None and tuple(add.shape) != shape:
        raise ValueError("add must have shape %s, got %s" % (shape, tuple(add.shape)))
    sizes = (distances.shape[0], math.prod(distances.shape[1:]))
    source = ("tm_distance_bias", (distances.data_ptr(), DISTANCES[distances.dtype]) + sizes, distances)
    return _run_bias(table, edges, add, source, shape)


def _extents(value, what):
    extents = (value,) if isinstance(value, int) else tuple(int(n) for n in value)
    if not 1 <= len(extents) <= 8:
        raise ValueError("%s must have 1 to 8 axes" % what)
    return extents


@functools.lru_cache(maxsize=1024)
def _grid(query, key, offset, metric, sampling):
    """(what the entry points take of a grid, but for the batch; queries; keys)."""
    ndim = len(query)
    if len(key) != ndim:
        raise ValueError("query_shape has %d axes, key_shape %d" % (ndim, len(key)))
    if min(query + key) < 0:
        raise ValueError("extents must not be negative, got %s and %s" % (query, key))
    offset = (offset,) + (0,) * (ndim - 1) if isinstance(offset, int) else offset
    if len(offset) != ndim:
        raise ValueError("query_offset must have %d coordinates, got %d" % (ndim, len(offset)))
    if metric not in BIAS_METRICS:
        raise ValueError("metric must be one of %s" % sorted(BIAS_METRICS))
    if metric == "offset" and (ndim != 1 or sampling is not None):
        raise ValueError("metric 'offset' is for sequences, without sampling")
    if sampling is not None:
        sampling = (sampling,) * ndim if isinstance(sampling, float) else sampling
        if len(sampling) != ndim:
            raise RuntimeError("sequence argument must have length equal to input rank")
    args = (ndim, _shape_array(query), _shape_array(key), _shape_array(offset), BIAS_METRICS[metric],
            _sampling_array(sampling, ndim))
    return args, math.prod(query), math.prod(key)


def relative_bias(table: torch.Tensor, edges: torch.Tensor, query_shape, key_shape, *, query_offset=0,
                  metric: str = "euclidean", sampling=None, add: Optional[torch.Tensor] = None) -> torch.Tensor:
    """A learned bias by buckets of the distance between a query's and a key's
    position, for attention over a sequence, an image or a volume:

        out[h, q, k] = table[number of edges <= D(q, k), h]  (+ add[..., h, q, k])

    ``query_shape``, ``key_shape``  extents of the grids of queries and keys (an
                int for a sequence); positions run in row-major order.
    ``query_offset``  coordinates of the first query (an int: along the first
                axis), as for one new token at the end of its sequence.
    ``metric``  "offset": the signed difference key - query of a sequence;
                "euclidean", "taxicab" or "chessboard": the library's distances,
                with ``sampling`` the spacing along each axis.
    ``table``, ``edges``  as for ``distance_bias``.
    ``add``     (*batch, heads, queries, keys), such as attention scores.

    Returns (heads, queries, keys) of the table's type, or the shape and type
    of ``add``.  Gradients flow to ``table`` (summed over the batch) and ``add``.
    """
    table, edges, add = _check_bias(table, edges, add)
    if sampling is not None:
        sampling = float(sampling) if isinstance(sampling, (int, float)) else tuple(float(s) for s in sampling)
    args, queries, keys = _grid(_extents(query_shape, "query_shape"), _extents(key_shape, "key_shape"),
                                query_offset if isinstance(query_offset, int) else tuple(int(n) for n in query_offset),
                                metric, sampling)
    shape, batch = (table.shape[1], queries, keys), 1
    if add is not None:
        tail, shape = shape, tuple(add.shape)
        if shape[-3:] != tail:
            raise ValueError("add must have shape (..., %d, %d, %d), got %s" % (tail + (shape,)))
        batch = math.prod(shape[:-3])
    return _run_bias(table, edges, add, ("tm_relative_bias", args + (batch,), None), shape)
