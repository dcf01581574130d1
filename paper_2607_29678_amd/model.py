"""Binding of ``include/toktier_model.h``: the operators next to the tokenizer, on both sides of a model.

``step_plan`` lays the tokens of a step out in a paged cache; ``token_scores`` and ``head_scores``
give the log probabilities of given tokens with entropy (and alternatives), from stored logits or
from hidden states and the head's weights; ``token_scores_grad`` and ``head_scores_grad`` are their
gradients.

Like the rest of the package the functions only check and marshal arguments; PyTorch is not
imported.  Tensors are device tensors with the attributes of torch's; outputs are the caller's.  The
calls enqueue on ``stream`` (a HIP stream handle as an int, None for the null stream) of the current
device, which has to be the tensors', and return at once.  The C calls trust the shapes they are told,
so every shape, type, stride and device is checked here; a mismatch raises ``ValueError``.
"""

import functools
import struct

from . import _lib

_NAMES = {"torch.float32": _lib.TT_F32, "torch.bfloat16": _lib.TT_BF16, "torch.float16": _lib.TT_F16, "torch.int32": "i32",
          "torch.int64": "i64", "torch.uint8": "u8"}
_F32, _I32, _I64, _U8 = _lib.TT_F32, "i32", "i64", "u8"
_codes = {}  # dtype -> its code (the types' names are long to make)


_known = _codes.get


def _code(dtype):
    code = _known(dtype)
    return _codes.setdefault(dtype, _NAMES.get(str(dtype))) if code is None else code


def _device(t, name):
    """Device of a call's first tensor.  The launch goes to the current device, so that has to be it."""
    device = t.get_device()
    if device < 0:
        raise ValueError("%s must be a device tensor, not on %s" % (name, t.device))
    current = _lib.load().tt_current_device()
    if device != current:
        raise ValueError("%s is on device %d, but device %d is current" % (name, device, current))
    return device


def _flat(t, name, code, shape, device):
    """Address of a contiguous tensor of this type and shape on this device; 0 for None."""
    if t is None:
        return 0
    if t.shape == shape and _known(t.dtype) == code and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    if t.shape != shape or _code(t.dtype) != code or t.get_device() != device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s device tensor of shape %s, on device %d with the others, not %s %s on %s"
                         % (name, {v: k for k, v in _NAMES.items()}[code], tuple(shape), device, t.dtype, tuple(t.shape),
                            t.device))
    return t.data_ptr()


def _matrix(t, name, device, dtype=None, shape=None):
    """(address, row stride) of a device matrix whose rows are contiguous and do not overlap."""
    if t.dim() != 2 or t.get_device() != device or (dtype is not None and t.dtype != dtype) or \
            (shape is not None and t.shape != shape):
        raise ValueError("%s must be a device matrix%s%s, on device %d with the others, not %s %s on %s"
                         % (name, "" if dtype is None else " of %s" % dtype, "" if shape is None else " of shape %s" % (shape,),
                            device, t.dtype, tuple(t.shape), t.device))
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
    code = _code(t.dtype)
    if code not in allowed:
        raise ValueError("%s has type %s, which this call does not take" % (name, t.dtype))
    return code


def _room(workspace, need, device):
    if workspace is None:
        if need > 0:
            raise ValueError("a workspace of %d bytes is needed" % need)
        return None, 0
    if _code(workspace.dtype) != _U8 or workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on device %d" % device)
    size, p = workspace.numel(), workspace.data_ptr()
    if size < need or p % 256:
        raise ValueError("workspace must hold %d bytes, aligned to 256: it has %d" % (need, size))
    return p, size


@functools.lru_cache(maxsize=256)
def _need(name, *sizes):
    """A workspace size: a function of sizes alone."""
    size = getattr(_lib.load(), name)(*sizes)
    if size < 0:
        raise _lib.TokTierError(int(size), name)
    return int(size)


# tt_step, packed as the compiler lays it out
_STEP = struct.Struct("@iii4xqqq15P")


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
    d, each, room, free = _device(cached, "cached"), cached.shape, slots.shape, free_pages.shape
    n = each[0]
    table, stride = _matrix(tables, "tables", d)
    width = tables.shape[1]
    if _code(tables.dtype) != _I32 or tables.shape[0] != n:
        raise ValueError("tables must be an int32 matrix of %d rows, not %s %s" % (n, tables.dtype, tuple(tables.shape)))
    if len(each) != 1 or len(room) != 1 or len(free) != 1:
        raise ValueError("cached, slots and free_pages must have one dimension")
    flat = _flat
    if not -0x80000000 <= page_size <= 0x7FFFFFFF:  # (0 and less the call itself refuses)
        raise ValueError("page_size %r does not fit 32 bits" % (page_size,))
    step = _STEP.pack(
        n, page_size, width, stride, room[0], free[0], flat(cached, "cached", _I32, each, d),
        flat(fresh, "fresh", _I32, each, d), flat(held, "held", _I32, each, d), flat(ids, "ids", _I32, room, d),
        flat(free_pages, "free_pages", _I32, free, d), flat(free_count, "free_count", _I64, (1,), d), table,
        flat(offsets, "offsets", _I32, (n + 1,), d), flat(lengths, "lengths", _I32, each, d),
        flat(pages, "pages", _I32, each, d), flat(slots, "slots", _I64, room, d), flat(positions, "positions", _I32, room, d),
        flat(requests, "requests", _I32, room, d), flat(targets, "targets", _I32, room, d),
        flat(result, "result", _I64, (2,), d))
    _lib.check(_lib.load().tt_step_plan(step, stream), "tt_step_plan")


def token_scores_workspace(rows, vocab, n_alt=0) -> int:
    """``tt_token_scores_workspace``: bytes of workspace that ``token_scores`` needs (0: none)."""
    return _need("tt_token_scores_workspace", rows, vocab, n_alt)


def token_scores(logits, targets, logprobs=None, stats=None, entropy=None, alt_ids=None, alt_logprobs=None, scale=1.0,
                 workspace=None, stream=None):
    """``tt_token_scores``: scores of rows of logits [rows, vocab] (float32, bfloat16 or float16).

    ``targets`` (int32 [rows] or None), ``logprobs``, ``entropy`` (float32 [rows]), ``stats``
    (float32 [rows, 2]) and ``alt_ids`` (int32), ``alt_logprobs`` (float32) [rows, k] for the ``k``
    best alternatives; outputs that are None are not computed.
    """
    d = _device(logits, "logits")
    p, stride = _matrix(logits, "logits", d)
    kind = _type_of(logits, "logits", (0, 1, 2))
    rows, vocab = logits.shape
    if (alt_ids is None) != (alt_logprobs is None):
        raise ValueError("alt_ids and alt_logprobs come together")
    k = 0 if alt_ids is None else alt_ids.shape[-1]
    room, size = _room(workspace, _need("tt_token_scores_workspace", rows, vocab, k), d)
    _lib.check(_lib.load().tt_token_scores(
        p, kind, rows, vocab, stride, scale, _flat(targets, "targets", _I32, (rows,), d),
        _flat(logprobs, "logprobs", _F32, (rows,), d), _flat(stats, "stats", _F32, (rows, 2), d),
        _flat(entropy, "entropy", _F32, (rows,), d), k, _flat(alt_ids, "alt_ids", _I32, (rows, k), d),
        _flat(alt_logprobs, "alt_logprobs", _F32, (rows, k), d), room, size, stream), "tt_token_scores")


def token_scores_grad(logits, targets, stats, entropy, grad_logprobs, grad_entropy, grad_logits, scale=1.0, stream=None):
    """``tt_token_scores_grad``: gradient with respect to the logits, into ``grad_logits`` (the
    logits' type and shape; may be the logits).  ``targets``, ``grad_logprobs`` and ``grad_entropy``
    may be None; ``entropy`` may be None with ``grad_entropy``."""
    d = _device(logits, "logits")
    p, stride = _matrix(logits, "logits", d)
    kind = _type_of(logits, "logits", (0, 1, 2))
    rows, vocab = logits.shape
    q, grad_stride = _matrix(grad_logits, "grad_logits", d, logits.dtype, (rows, vocab))
    one = (rows,)
    _lib.check(_lib.load().tt_token_scores_grad(
        p, kind, rows, vocab, stride, scale, _flat(targets, "targets", _I32, one, d),
        _flat(stats, "stats", _F32, (rows, 2), d), _flat(entropy, "entropy", _F32, one, d),
        _flat(grad_logprobs, "grad_logprobs", _F32, one, d), _flat(grad_entropy, "grad_entropy", _F32, one, d),
        q, grad_stride, stream), "tt_token_scores_grad")


def head_scores_workspace(rows, vocab, width) -> int:
    """``tt_head_scores_workspace``: bytes of workspace that ``head_scores`` needs."""
    return _need("tt_head_scores_workspace", rows, vocab, width)


def _head(hidden, weight, device):
    h, h_stride = _matrix(hidden, "hidden", device)
    w, w_stride = _matrix(weight, "weight", device, hidden.dtype)
    kind = _type_of(hidden, "hidden", (1, 2))
    if weight.shape[1] != hidden.shape[1]:
        raise ValueError("hidden has rows of %d entries, weight of %d" % (hidden.shape[1], weight.shape[1]))
    return (h, h_stride, w, w_stride, kind, hidden.shape[0], weight.shape[0], hidden.shape[1])


def head_scores(hidden, weight, targets, logprobs=None, stats=None, entropy=None, scale=1.0, workspace=None, stream=None):
    """``tt_head_scores``: the scores of ``hidden @ weight.T`` (bfloat16 or float16) without storing it;
    arguments as those of ``token_scores``."""
    d = _device(hidden, "hidden")
    head = _head(hidden, weight, d)
    rows, vocab, width = head[5:]
    room, size = _room(workspace, _need("tt_head_scores_workspace", rows, vocab, width), d)
    _lib.check(_lib.load().tt_head_scores(
        *head, scale, _flat(targets, "targets", _I32, (rows,), d), _flat(logprobs, "logprobs", _F32, (rows,), d),
        _flat(stats, "stats", _F32, (rows, 2), d), _flat(entropy, "entropy", _F32, (rows,), d), room, size, stream),
        "tt_head_scores")


def head_scores_grad_workspace(rows, vocab, width, ample=True) -> int:
    """``tt_head_scores_grad_workspace``: the least bytes of workspace, or (``ample``) those up to
    which more room helps."""
    return _need("tt_head_scores_grad_workspace", rows, vocab, width, 1 if ample else 0)


def head_scores_grad(hidden, weight, targets, stats, entropy, grad_logprobs, grad_entropy, grad_hidden, grad_weight,
                     scale=1.0, workspace=None, stream=None):
    """``tt_head_scores_grad``: gradients with respect to ``hidden`` and ``weight`` (either output may
    be None); the other arguments as those of ``token_scores_grad``."""
    d = _device(hidden, "hidden")
    head = _head(hidden, weight, d)
    rows, vocab, width = head[5:]
    gh = (None, width) if grad_hidden is None else _matrix(grad_hidden, "grad_hidden", d, hidden.dtype, (rows, width))
    gw = (None, width) if grad_weight is None else _matrix(grad_weight, "grad_weight", d, hidden.dtype, (vocab, width))
    one = (rows,)
    room, size = _room(workspace, _need("tt_head_scores_grad_workspace", rows, vocab, width, 0), d)
    _lib.check(_lib.load().tt_head_scores_grad(
        *head, scale, _flat(targets, "targets", _I32, one, d), _flat(stats, "stats", _F32, (rows, 2), d),
        _flat(entropy, "entropy", _F32, one, d), _flat(grad_logprobs, "grad_logprobs", _F32, one, d),
        _flat(grad_entropy, "grad_entropy", _F32, one, d), *gh, *gw, room, size, stream), "tt_head_scores_grad")
