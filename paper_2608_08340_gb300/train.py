"""Operators that train a query encoder against an index.

A large encoder's search results (``Index.search``: ids and scores) teach a small
one: token rows are looked up, pooled into a query, scored against the chunks, and
the scores are held to the results.  One training step:

    hidden = embed_lookup(table, ids, scale)                 # ids: -1 where padded
    query, mean = embed_pool_train(hidden, mask)
    loss, dlogits = distill_loss(query @ E.T, t_ids, t_scores, temperature=0.05)
    dhidden = embed_pool_grad(dlogits @ E, mean, mask)
    dtable = embed_lookup_grad(dhidden, ids, vocab, scale)

Every call enqueues hand-written kernels of liboprag.so on `stream` (a
torch.cuda.Stream; default: the current one) and returns tensors that belong to that
stream.  Inputs have to be ready on it; they may be dropped behind the call, their memory
is not given away before that stream has got past it.  Rows that are not laid out as a
kernel reads them are copied on that stream first.

Under torch's automatic differentiation embed_lookup's rows, embed_pool_train's out and
distill_loss's loss lead back to a table, hidden states and logits that require a
gradient, through the calls above (so `loss.mean().backward()` does the rest of the
step); the teacher's results, the weight and the mean are constants there, and the two
gradients have no derivative of their own.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from . import _lib
from ._lib import check
from .index import _DT

_IDS = {torch.int32: 0, torch.int64: 1}
_MASKS = (torch.uint8, torch.bool)
# torch.cuda.current_device's answer, and current_stream(device).cuda_stream without
# its Stream object.  The host's share of a small call is its time: 3 of 10 us are
# these checks, 4 the result tensor, 3 the C call.
_current_device = torch._C._cuda_getDevice
_stream = torch._C._cuda_getCurrentRawStream


def _check_device(first: torch.Tensor, second: torch.Tensor, third=None) -> int:
    """The index of the device of all tensors: the current one."""
    at = first.get_device()
    if (at >= 0 and at == second.get_device() and at == _current_device()
            and (third is None or third.get_device() == at)):
        return at
    for t in (second, third):
        if t is not None and t.get_device() != at:
            raise ValueError(f"tensors are on {first.device} and {t.device}")
    if at < 0:
        raise ValueError("tensors must be on the GPU")
    raise ValueError(f"tensors are on {first.device}, which is not the current device")


_functions = {}


def _call(name: str, *args) -> None:
    function = _functions.get(name)
    if function is None:
        function = _functions.setdefault(name, getattr(_lib.load(), name))
    rc = function(*args)
    if rc != 0:
        check(rc)


def _on(stream, call, *args):
    """call(*args) with `stream` current; its tensors, which may be another stream's, are
    kept for it."""
    with torch.cuda.stream(stream):
        result = call(*args)
    for t in args:
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
    return result


def _tracked(t: torch.Tensor) -> bool:
    return t.requires_grad and torch.is_grad_enabled()


def _written(out: torch.Tensor) -> None:
    """Tells torch that a given `out` changed: a graph that needs its former values
    refuses to go on without them."""
    if not out.is_inference():
        torch.autograd.graph.increment_version(out)


class _Lookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, rows, ids, scale):
        ctx.save_for_backward(ids)
        ctx.table = (table.shape[0], scale, table.dtype)
        ctx.mark_dirty(rows)
        return rows

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        ids, = ctx.saved_tensors
        if ids.dim() == 0:
            ids, grad = ids.unsqueeze(0), grad.unsqueeze(0)
        return embed_lookup_grad(grad, ids, *ctx.table), None, None, None


class _Pool(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, out, mean, mask):
        ctx.save_for_backward(mean, mask)
        ctx.dtype = hidden.dtype
        ctx.mark_dirty(out)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        return embed_pool_grad(grad, *ctx.saved_tensors, ctx.dtype), None, None, None


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, loss, teacher_ids, teacher_scores, temperature):
        ctx.save_for_backward(logits, teacher_ids, teacher_scores)
        ctx.temperature = temperature
        ctx.mark_dirty(loss)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        _, dlogits = distill_loss(*ctx.saved_tensors, ctx.temperature, grad)
        return dlogits, None, None, None, None


def _check_sizes(*sizes: int) -> None:
    """The C ABI takes these sizes in 32 bits, and ctypes would cut them off."""
    if max(sizes) > 0x7FFFFFFF:
        raise ValueError(f"a size of {max(sizes)} is outside [0, 2^31)")


def _whole(t: torch.Tensor) -> torch.Tensor:
    """t, contiguous and on 16 bytes; a copy where it is not."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _strides(t: torch.Tensor) -> list[int]:
    """Strides of the dimensions before the last; 0 where there is one entry."""
    return [s if n > 1 else 0 for s, n in zip(t.stride()[:-1], t.shape[:-1])]


def _rows_fit(t: torch.Tensor) -> bool:
    """Rows of the last dimension are contiguous and start on 16 bytes (a row of a
    contiguous tensor does where the dimension is one that the kernels take)."""
    if t.is_contiguous():
        return t.data_ptr() % 16 == 0
    step = 16 // t.element_size()
    return (t.stride(-1) == 1 and t.data_ptr() % 16 == 0
            and all(s % step == 0 for s in _strides(t)))


def _rows_apart(t: torch.Tensor) -> bool:
    """Rows of a matrix are contiguous and do not overlap."""
    return ((t.shape[1] == 1 or t.stride(1) == 1)
            and (t.shape[0] == 1 or t.stride(0) >= t.shape[1]))


def embed_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0,
                 out_dtype: torch.dtype | None = None, stream=None, out=None) -> torch.Tensor:
    """Rows of an embedding table: scale * table[ids], in out_dtype (default the table's).

    table: (vocab, dim) bfloat16 or float32, dim a multiple of 8; ids: int32 or int64
    of any shape, an id outside [0, vocab) gives a zero row (padding).  Returns
    ids.shape + (dim,)."""
    if stream is not None:
        return _on(stream, embed_lookup, table, ids, scale, out_dtype, None, out)
    rows = table.shape
    if len(rows) != 2 or table.dtype not in _DT:
        raise ValueError("table must be a 2-D bfloat16 or float32 tensor")
    if ids.dtype not in _IDS:
        raise ValueError("ids must be int32 or int64")
    vocab, dim = rows
    _check_sizes(dim)
    device = _check_device(table, ids)
    shape = (*ids.shape, dim)
    given = out is not None
    if not given:
        out_dtype = out_dtype or table.dtype
        if out_dtype not in _DT:
            raise ValueError("out_dtype must be bfloat16 or float32")
        out = torch.empty(shape, dtype=out_dtype, device=device)
    elif (tuple(out.shape) != shape or out.dtype not in _DT or not out.is_contiguous()
          or out.get_device() != device or out_dtype not in (None, out.dtype)):
        raise ValueError(f"out must be a contiguous {shape} tensor")
    stride = dim
    if not _rows_fit(table) or (vocab > 1 and table.stride(0) < dim):
        table = table.clone(memory_format=torch.contiguous_format)
    elif vocab > 1:
        stride = table.stride(0)
    ids = ids.contiguous()
    _call("oprag_embed_lookup",
          table.data_ptr(), _DT[table.dtype], vocab, dim, stride, ids.data_ptr(), _IDS[ids.dtype],
          ids.numel(), scale, out.data_ptr(), _DT[out.dtype], _stream(device))
    if given:
        _written(out)
    return _Lookup.apply(table, out, ids, scale) if _tracked(table) else out


def embed_lookup_grad(grad: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0,
                      out_dtype: torch.dtype = torch.float32, stream=None,
                      out=None) -> torch.Tensor:
    """Gradient of embed_lookup for its table: (vocab, dim) in out_dtype, row v
    scale times the sum of grad over the tokens whose id is v (float32 sums in an
    order given by the ids; zeros for a row without tokens).  Padding is best given
    as -1 (ids.masked_fill(ids == pad, -1)): the tokens of a padding id of the table are
    added up like any other's, in up to twice the time.

    grad: ids.shape + (dim,) bfloat16 or float32; it may be a broadcast, such as
    rows.unsqueeze(1).expand(-1, tokens, -1) where all tokens of a text share a row:
    it is read as it lies.  ids as for embed_lookup, with at least one dimension."""
    if stream is not None:
        return _on(stream, embed_lookup_grad, grad, ids, vocab, scale, out_dtype, None, out)
    if grad.dtype not in _DT or ids.dtype not in _IDS:
        raise ValueError("grad must be bfloat16 or float32, ids int32 or int64")
    if ids.dim() < 1 or grad.dim() != ids.dim() + 1 or grad.shape[:-1] != ids.shape:
        raise ValueError("grad must have the shape of ids and one dimension more")
    if out_dtype not in _DT:
        raise ValueError("out_dtype must be bfloat16 or float32")
    dim, count = grad.shape[-1], ids.numel()
    _check_sizes(dim)
    device = _check_device(grad, ids)
    need = ctypes.c_int64()
    _call("oprag_embed_lookup_grad_workspace", count, vocab, dim, ctypes.byref(need))
    given = out is not None
    if not given:
        out = torch.empty((vocab, dim), dtype=out_dtype, device=device)
    elif (tuple(out.shape) != (vocab, dim) or out.dtype != out_dtype
          or not out.is_contiguous() or out.get_device() != device):
        raise ValueError(f"out must be a contiguous {(vocab, dim)} tensor of {out_dtype}")
    ids = ids.contiguous()
    if grad.dim() == 2:
        grad = grad.unsqueeze(0)
    elif grad.dim() > 3:
        grad = grad.flatten(0, -3)
    if not _rows_fit(grad):
        grad = grad.clone(memory_format=torch.contiguous_format)
    work = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
    _call("oprag_embed_lookup_grad",
          grad.data_ptr(), _DT[grad.dtype], grad.shape[0], grad.shape[1], dim, *_strides(grad),
          ids.data_ptr(), _IDS[ids.dtype], vocab, scale, out.data_ptr(), _DT[out_dtype],
          None if work is None else work.data_ptr(), need.value, _stream(device))
    if given:
        _written(out)
    return out


def _hidden_mask(mask: torch.Tensor, batch: int) -> torch.Tensor:
    if mask.dim() != 2 or mask.shape[0] != batch or mask.dtype not in _MASKS:
        raise ValueError("mask must be (batch, tokens) bool or uint8")
    return mask.contiguous()


def embed_pool_train(hidden: torch.Tensor, mask: torch.Tensor,
                     out_dtype: torch.dtype = torch.bfloat16, stream=None):
    """embed_pool that keeps what its gradient needs: (out, mean), mean the float32
    (batch, dim) pooled rows before normalisation."""
    if stream is not None:
        return _on(stream, embed_pool_train, hidden, mask, out_dtype)
    if hidden.dim() != 3 or hidden.dtype not in _DT:
        raise ValueError("hidden must be a 3-D bfloat16 or float32 tensor")
    if out_dtype not in _DT:
        raise ValueError("out_dtype must be bfloat16 or float32")
    b, t, d = hidden.shape
    _check_sizes(b, t, d)
    device = _check_device(hidden, mask)
    mask = _hidden_mask(mask, b)
    if mask.shape[1] != t:
        raise ValueError("mask must be (batch, tokens)")
    hidden = _whole(hidden)
    out = torch.empty((b, d), dtype=out_dtype, device=device)
    mean = torch.empty((b, d), dtype=torch.float32, device=device)
    _call("oprag_embed_pool_train",
          hidden.data_ptr(), _DT[hidden.dtype], b, t, d, mask.data_ptr(), out.data_ptr(),
          _DT[out_dtype], mean.data_ptr(), _stream(device))
    return (_Pool.apply(hidden, out, mean, mask) if _tracked(hidden) else out), mean


def embed_pool_grad(grad: torch.Tensor, mean: torch.Tensor, mask: torch.Tensor,
                    dtype: torch.dtype = torch.bfloat16, per_token: bool = True,
                    stream=None) -> torch.Tensor:
    """Gradient of embed_pool for its hidden states, (batch, tokens, dim) in dtype
    (zeros for padding); with per_token=False (batch, dim), the row that each of a
    text's real tokens has.

    grad: (batch, dim) gradient of embed_pool_train's out; mean: its second result;
    mask: the mask that it was given."""
    if stream is not None:
        return _on(stream, embed_pool_grad, grad, mean, mask, dtype, per_token)
    if grad.dim() != 2 or grad.dtype not in _DT:
        raise ValueError("grad must be a 2-D bfloat16 or float32 tensor")
    if mean.shape != grad.shape or mean.dtype != torch.float32:
        raise ValueError("mean must be float32 and have the shape of grad")
    if dtype not in _DT:
        raise ValueError("dtype must be bfloat16 or float32")
    b, d = grad.shape
    _check_sizes(b, d, *mask.shape)
    device = _check_device(grad, mean, mask)
    mask = _hidden_mask(mask, b)
    t = mask.shape[1]
    grad, mean = _whole(grad), _whole(mean)
    out = torch.empty((b, t, d) if per_token else (b, d), dtype=dtype, device=device)
    _call("oprag_embed_pool_grad",
          grad.data_ptr(), _DT[grad.dtype], mean.data_ptr(), b, t, d, mask.data_ptr(),
          out.data_ptr(), _DT[dtype], int(per_token), _stream(device))
    return out


def distill_loss(logits: torch.Tensor, teacher_ids: torch.Tensor, teacher_scores: torch.Tensor,
                 temperature: float = 1.0, weight: torch.Tensor | None = None, grad: bool = True,
                 stream=None, out=None):
    """Divergence of a student's scores from a teacher's search results, and its
    gradient: (loss, grad).

    logits: (q, n) bfloat16 or float32, the student's scores of the n chunks, -inf or
    the dtype's lowest value where a chunk is hidden from a row; teacher_ids int64 and
    teacher_scores float32 (q, k), k <= 256, as Index.search returns them (an id outside
    [0, n), a score of -inf or a hidden chunk: no result).  With
    t = softmax(teacher_scores / temperature) over the results and
    p = softmax(logits / temperature),

        loss[i] = sum_j t_j (ln t_j - ln p[id_j])      float32 (q,), not weighted
        grad    = weight[i] / temperature * (p - t)    (q, n) in the logits' dtype

    weight: (q,) float32, default 1 for every row.  A row without results has loss 0
    and no gradient.  grad=False: (loss, None).  out: where the gradient goes, a (q, n)
    tensor with contiguous rows; it may be logits, or lie apart from its rows.

    p and t carry the device's approximate exponential: some (4 |x| + 4 mean |x| + 24) 2^-24
    of themselves for x = (logits - max) / temperature, up to twice what expf leaves.  The
    same call gives the same bits; a row's last bits may depend on q."""
    if stream is not None:
        return _on(stream, distill_loss, logits, teacher_ids, teacher_scores, temperature, weight,
                   grad, None, out)
    shape, results = logits.shape, teacher_ids.shape
    if len(shape) != 2 or logits.dtype not in _DT:
        raise ValueError("logits must be a 2-D bfloat16 or float32 tensor")
    q, n = shape
    if (len(results) != 2 or results[0] != q or teacher_scores.shape != results
            or teacher_ids.dtype != torch.int64 or teacher_scores.dtype != torch.float32):
        raise ValueError("teacher_ids (int64) and teacher_scores (float32) must be (q, k)")
    _check_sizes(q, n, results[1])
    device = _check_device(logits, teacher_ids, teacher_scores)
    if weight is not None:
        if weight.shape != shape[:1] or weight.dtype != torch.float32:
            raise ValueError("weight must be (q,) float32")
        _check_device(logits, weight)
        weight = weight.contiguous()
    stride = out_stride = n
    whole, given = logits.is_contiguous(), grad and out is not None
    if not grad:
        out = None
    elif out is None:
        out = (torch.empty_like(logits) if whole
               else torch.empty(shape, dtype=logits.dtype, device=device))
    elif (out.shape != shape or out.dtype != logits.dtype or not _rows_apart(out)
          or out.get_device() != device):
        raise ValueError("out must be like logits, with contiguous rows")
    elif q > 1:
        out_stride = out.stride(0)
    if not whole:
        if not _rows_apart(logits):
            logits = logits.clone(memory_format=torch.contiguous_format)
        elif q > 1:
            stride = logits.stride(0)
    teacher_ids, teacher_scores = teacher_ids.contiguous(), teacher_scores.contiguous()
    loss = torch.empty(q, dtype=torch.float32, device=device)
    _call("oprag_distill",
          logits.data_ptr(), _DT[logits.dtype], stride, q, n, teacher_ids.data_ptr(),
          teacher_scores.data_ptr(), results[1], temperature,
          None if weight is None else weight.data_ptr(), loss.data_ptr(),
          None if out is None else out.data_ptr(), out_stride, _stream(device))
    if _tracked(logits):
        loss = _Distill.apply(logits, loss, teacher_ids, teacher_scores, temperature)
    if given:                             # (behind the graph's note of the scores)
        _written(out)
    return loss, out
