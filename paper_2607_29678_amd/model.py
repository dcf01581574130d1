"""Binding of ``include/toktier_model.h``: the operators next to the tokenizer, on both sides of a model.

``step_plan`` lays the tokens of a step out in a paged cache; ``token_scores`` and ``head_scores``
give the log probabilities of given tokens with entropy (and alternatives), from stored logits or
from hidden states and the head's weights; ``token_scores_grad`` and ``head_scores_grad`` are their
gradients.

Like the rest of the package the functions only check and marshal arguments; PyTorch is not
imported.  Tensors are device tensors with the attributes of torch's; outputs are the caller's.  The
calls enqueue on ``stream`` (a HIP stream handle as an int, None for the null stream), which has
to belong to the tensors' device, and return at once.  The C calls trust the shapes they are told,
so every shape, type and stride is checked here; a mismatch raises ``ValueError``.
"""

import ctypes

from . import _lib

_TYPES = {"torch.float32": _lib.TT_F32, "torch.bfloat16": _lib.TT_BF16, "torch.float16": _lib.TT_F16}


def _same_device(first, *others):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("tensors are on different devices: %s and %s" % (first.device, t.device))


def _flat(t, name, dtype, shape):
    """Address of a contiguous device tensor of this type and shape; None for None."""
    if t is None:
        return None
    if str(t.dtype) != dtype or tuple(t.shape) != shape or not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s device tensor of shape %s, not %s %s on %s"
                         % (name, dtype, shape, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _matrix(t, name, dtype=None, shape=None):
    """(address, row stride) of a device matrix whose rows are contiguous and do not overlap."""
    if t.dim() != 2 or not t.is_cuda or (dtype is not None and t.dtype != dtype) or \
            (shape is not None and tuple(t.shape) != shape):
        raise ValueError("%s must be a device matrix%s%s, not %s %s on %s"
                         % (name, "" if dtype is None else " of %s" % dtype, "" if shape is None else " of shape %s" % (shape,),
                            t.dtype, tuple(t.shape), t.device))
    rows, cols = t.shape
    stride, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError("the rows of %s must be contiguous" % name)
    if rows <= 1:
        stride = max(stride, cols)
    if stride < cols:
        raise ValueError("the rows of %s overlap" % name)
    return t.data_ptr(), stride


def _type_of(t, name, allowed):
    code = _TYPES.get(str(t.dtype))
    if code not in allowed:
        raise ValueError("%s has type %s, which this call does not take" % (name, t.dtype))
    return code


def _room(workspace, need):
    if need <= 0 and workspace is None:
        return None, 0
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous() or str(workspace.dtype) != "torch.uint8":
        raise ValueError("workspace must be a contiguous uint8 device tensor of at least %d bytes" % need)
    if workspace.numel() < need or workspace.data_ptr() % 256:
        raise ValueError("workspace must hold %d bytes, aligned to 256: it has %d" % (need, workspace.numel()))
    return workspace.data_ptr(), workspace.numel()


def _need(size):
    if size < 0:
        raise _lib.TokTierError(int(size), "workspace size")
    return int(size)


def step_plan(cached, fresh, tables, free_pages, free_count, page_size, offsets, lengths, pages, slots, positions, requests,
              result, held=None, ids=None, targets=None, stream=None):
    """``tt_step_plan``: the plan of a step of ``len(cached)`` requests.

    ``cached``, ``fresh``, ``held``, ``offsets`` (one entry more), ``lengths`` and ``pages`` are int32
    of one entry a request; ``tables`` is an int32 matrix of one row a request, updated in place;
    ``free_pages`` an int32 stack of which ``free_count`` (int64, one entry) entries are in use;
    ``slots`` (int64), ``positions``, ``requests``, ``ids`` and ``targets`` (int32) have one entry a
    token, as many as the step may hold; ``result`` (int64, two entries) receives the number of
    tokens and the free pages left, or a negative error code and the count as it was.
    """
    n, room = len(cached), len(slots)
    _same_device(cached, fresh, tables, free_pages, free_count, offsets, lengths, pages, slots, positions, requests, result,
                 held, ids, targets)
    table, stride = _matrix(tables, "tables")
    if str(tables.dtype) != "torch.int32" or tables.shape[0] != n:
        raise ValueError("tables must be an int32 matrix of %d rows, not %s %s" % (n, tables.dtype, tuple(tables.shape)))
    i32, i64 = "torch.int32", "torch.int64"
    step = _lib.Step(n, page_size, tables.shape[1], stride, room, len(free_pages),
                     _flat(cached, "cached", i32, (n,)), _flat(fresh, "fresh", i32, (n,)), _flat(held, "held", i32, (n,)),
                     _flat(ids, "ids", i32, (room,)), _flat(free_pages, "free_pages", i32, (len(free_pages),)),
                     _flat(free_count, "free_count", i64, (1,)), table, _flat(offsets, "offsets", i32, (n + 1,)),
                     _flat(lengths, "lengths", i32, (n,)), _flat(pages, "pages", i32, (n,)),
                     _flat(slots, "slots", i64, (room,)), _flat(positions, "positions", i32, (room,)),
                     _flat(requests, "requests", i32, (room,)), _flat(targets, "targets", i32, (room,)),
                     _flat(result, "result", i64, (2,)))
    _lib.check(_lib.load().tt_step_plan(ctypes.byref(step), stream), "tt_step_plan")


def token_scores_workspace(rows, vocab, n_alt=0) -> int:
    """``tt_token_scores_workspace``: bytes of workspace that ``token_scores`` needs (0: none)."""
    return _need(_lib.load().tt_token_scores_workspace(rows, vocab, n_alt))


def token_scores(logits, targets, logprobs=None, stats=None, entropy=None, alt_ids=None, alt_logprobs=None, scale=1.0,
                 workspace=None, stream=None):
    """``tt_token_scores``: scores of rows of logits [rows, vocab] (float32, bfloat16 or float16).

    ``targets`` (int32 [rows] or None), ``logprobs``, ``entropy`` (float32 [rows]), ``stats``
    (float32 [rows, 2]) and ``alt_ids`` (int32), ``alt_logprobs`` (float32) [rows, k] for the ``k``
    best alternatives; outputs that are None are not computed.
    """
    p, stride = _matrix(logits, "logits")
    kind = _type_of(logits, "logits", (0, 1, 2))
    rows, vocab = logits.shape
    _same_device(logits, targets, logprobs, stats, entropy, alt_ids, alt_logprobs, workspace)
    if (alt_ids is None) != (alt_logprobs is None):
        raise ValueError("alt_ids and alt_logprobs come together")
    k = 0 if alt_ids is None else int(alt_ids.shape[-1])
    f32 = "torch.float32"
    lib = _lib.load()
    room, size = _room(workspace, _need(lib.tt_token_scores_workspace(rows, vocab, k)))
    _lib.check(lib.tt_token_scores(
        p, kind, rows, vocab, stride, scale, _flat(targets, "targets", "torch.int32", (rows,)),
        _flat(logprobs, "logprobs", f32, (rows,)), _flat(stats, "stats", f32, (rows, 2)),
        _flat(entropy, "entropy", f32, (rows,)), k, _flat(alt_ids, "alt_ids", "torch.int32", (rows, k)),
        _flat(alt_logprobs, "alt_logprobs", f32, (rows, k)), room, size, stream), "tt_token_scores")


def token_scores_grad(logits, targets, stats, entropy, grad_logprobs, grad_entropy, grad_logits, scale=1.0, stream=None):
    """``tt_token_scores_grad``: gradient with respect to the logits, into ``grad_logits`` (the
    logits' type and shape; may be the logits).  ``targets``, ``grad_logprobs`` and ``grad_entropy``
    may be None; ``entropy`` may be None with ``grad_entropy``."""
    p, stride = _matrix(logits, "logits")
    kind = _type_of(logits, "logits", (0, 1, 2))
    rows, vocab = logits.shape
    q, grad_stride = _matrix(grad_logits, "grad_logits", logits.dtype, (rows, vocab))
    _same_device(logits, targets, stats, entropy, grad_logprobs, grad_entropy, grad_logits)
    f32 = "torch.float32"
    _lib.check(_lib.load().tt_token_scores_grad(
        p, kind, rows, vocab, stride, scale, _flat(targets, "targets", "torch.int32", (rows,)),
        _flat(stats, "stats", f32, (rows, 2)), _flat(entropy, "entropy", f32, (rows,)),
        _flat(grad_logprobs, "grad_logprobs", f32, (rows,)), _flat(grad_entropy, "grad_entropy", f32, (rows,)),
        q, grad_stride, stream), "tt_token_scores_grad")


def head_scores_workspace(rows, vocab, width) -> int:
    """``tt_head_scores_workspace``: bytes of workspace that ``head_scores`` needs."""
    return _need(_lib.load().tt_head_scores_workspace(rows, vocab, width))


def _head(hidden, weight):
    h, h_stride = _matrix(hidden, "hidden")
    w, w_stride = _matrix(weight, "weight", hidden.dtype)
    kind = _type_of(hidden, "hidden", (1, 2))
    if weight.shape[1] != hidden.shape[1]:
        raise ValueError("hidden has rows of %d entries, weight of %d" % (hidden.shape[1], weight.shape[1]))
    return (h, h_stride, w, w_stride, kind, hidden.shape[0], weight.shape[0], hidden.shape[1])


def head_scores(hidden, weight, targets, logprobs=None, stats=None, entropy=None, scale=1.0, workspace=None, stream=None):
    """``tt_head_scores``: the scores of ``hidden @ weight.T`` (bfloat16 or float16) without storing it;
    arguments as those of ``token_scores``."""
    head = _head(hidden, weight)
    rows, vocab, width = head[5:]
    _same_device(hidden, weight, targets, logprobs, stats, entropy, workspace)
    f32 = "torch.float32"
    lib = _lib.load()
    room, size = _room(workspace, _need(lib.tt_head_scores_workspace(rows, vocab, width)))
    _lib.check(lib.tt_head_scores(
        *head, scale, _flat(targets, "targets", "torch.int32", (rows,)), _flat(logprobs, "logprobs", f32, (rows,)),
        _flat(stats, "stats", f32, (rows, 2)), _flat(entropy, "entropy", f32, (rows,)), room, size, stream), "tt_head_scores")


def head_scores_grad_workspace(rows, vocab, width, ample=True) -> int:
    """``tt_head_scores_grad_workspace``: the least bytes of workspace, or (``ample``) those up to
    which more room helps."""
    return _need(_lib.load().tt_head_scores_grad_workspace(rows, vocab, width, int(bool(ample))))


def head_scores_grad(hidden, weight, targets, stats, entropy, grad_logprobs, grad_entropy, grad_hidden, grad_weight,
                     scale=1.0, workspace=None, stream=None):
    """``tt_head_scores_grad``: gradients with respect to ``hidden`` and ``weight`` (either output may
    be None); the other arguments as those of ``token_scores_grad``."""
    head = _head(hidden, weight)
    rows, vocab, width = head[5:]
    _same_device(hidden, weight, targets, stats, entropy, grad_logprobs, grad_entropy, grad_hidden, grad_weight, workspace)
    gh = (None, width) if grad_hidden is None else _matrix(grad_hidden, "grad_hidden", hidden.dtype, (rows, width))
    gw = (None, width) if grad_weight is None else _matrix(grad_weight, "grad_weight", hidden.dtype, (vocab, width))
    f32 = "torch.float32"
    lib = _lib.load()
    room, size = _room(workspace, _need(lib.tt_head_scores_grad_workspace(rows, vocab, width, 0)))
    _lib.check(lib.tt_head_scores_grad(
        *head, scale, _flat(targets, "targets", "torch.int32", (rows,)), _flat(stats, "stats", f32, (rows, 2)),
        _flat(entropy, "entropy", f32, (rows,)), _flat(grad_logprobs, "grad_logprobs", f32, (rows,)),
        _flat(grad_entropy, "grad_entropy", f32, (rows,)), *gh, *gw, room, size, stream), "tt_head_scores_grad")
