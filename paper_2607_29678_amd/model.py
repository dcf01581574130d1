"""Binding of ``include/toktier_model.h``: the operators next to the tokenizer, on both sides of a model.

``step_plan`` lays the tokens of a step out in a paged cache, ``cache_append`` writes their keys and
values there (rotated by their positions) and ``cache_attention`` reads them; ``adjust_logits`` applies
penalties, biases and masks, with its gradient ``adjust_logits_grad``; ``token_scores`` and ``head_scores``
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


def _entries(t, name):
    """Entries of a tensor of one dimension."""
    shape = t.shape
    if len(shape) != 1:
        raise ValueError("%s must have one dimension, not shape %s" % (name, tuple(shape)))
    return shape[0]


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


# tt_cache, tt_attention and tt_adjustment, packed the same way
_CACHE = struct.Struct("@iiiiqqqqPP")
_ATTENTION = struct.Struct("@iiqqiiifqq6P")
_ADJUSTMENT = struct.Struct("@iiqqqqqq11P")


def _heads(t, name, device, dtype, tokens=None, heads=None, dim=None):
    """(address, row stride) of a device tensor [tokens, heads, dim] whose rows are contiguous and do not overlap."""
    shape = t.shape
    if len(shape) != 3 or t.dtype != dtype or t.get_device() != device or (tokens is not None and shape[0] != tokens) or \
            (heads is not None and shape[1] != heads) or (dim is not None and shape[2] != dim):
        raise ValueError("%s must be a %s tensor of [tokens%s, heads%s, dim%s] on device %d with the others, not %s %s on %s"
                         % (name, dtype, "" if tokens is None else " = %d" % tokens, "" if heads is None else " = %d" % heads,
                            "" if dim is None else " = %d" % dim, device, t.dtype, tuple(shape), t.device))
    row = _row_stride(shape, t.stride())
    if row < 0:
        raise ValueError("the rows of %s %s" % (name, "must be contiguous" if row == -1 else "overlap"))
    return t.data_ptr(), row


@functools.lru_cache(maxsize=256)
def _row_stride(shape, strides):
    """Distance of the rows [heads, dim] of a tensor of this shape and these strides: a function of them alone.
    -1: the rows are not contiguous; -2: they overlap."""
    (n, h, d), (row, head, step) = shape, strides
    if (d > 1 and step != 1) or (h > 1 and head != d):
        return -1
    if n <= 1:
        row = max(row, h * d)
    return row if row >= h * d else -2


@functools.lru_cache(maxsize=64)
def _cache_layout(shape, strides):
    """The sizes and strides of tt_cache for tensors of this shape and these strides: a function of them alone."""
    pages, page_size, heads, dim = shape
    if dim > 1 and strides[3] != 1:
        raise ValueError("the vectors of a cache must be contiguous")
    if page_size > 0x7FFFFFFF or heads > 0x7FFFFFFF or dim > 0x7FFFFFFF:
        raise ValueError("a cache of shape %s is too large" % (tuple(shape),))
    # no two vectors of a cache share elements: from the narrowest stride up, each is at least what lies below it
    below = dim
    for stride, size in sorted(zip(strides[:3], shape[:3])):
        if size > 1:
            if stride < below:
                raise ValueError("vectors of the cache overlap")
            below = stride * (size - 1) + below
    stride = [0 if n <= 1 else s for s, n in zip(strides, shape)]  # (one page, slot or head: its stride means nothing)
    return page_size, heads, dim, pages, stride[0], stride[1], stride[2]


def _cache(keys, values):
    """tt_cache of two tensors [pages, page_size, heads, dim] of the same strides; (packed, device)."""
    d = _device(keys, "key_cache")
    kind = _type_of(keys, "key_cache", (1, 2))
    shape, strides = keys.shape, keys.stride()
    if len(shape) != 4 or values.shape != shape or values.dtype != keys.dtype or values.get_device() != d:
        raise ValueError("key_cache and value_cache must be two tensors of [pages, page_size, heads, dim], not %s %s and %s %s on %s"
                         % (keys.dtype, tuple(shape), values.dtype, tuple(values.shape), values.device))
    if values.stride() != strides:
        raise ValueError("key_cache and value_cache must have the same strides")
    return _CACHE.pack(kind, *_cache_layout(shape, strides), keys.data_ptr(), values.data_ptr()), d


def cache_append(keys, values, key_cache, value_cache, slots, positions=None, frequencies=None, interleaved=False, queries=None,
                 rotated=None, stream=None):
    """``tt_cache_append``: keys and values of a step's tokens into their slots of a paged cache.

    ``keys`` and ``values`` are [tokens, heads, dim] (views of one projection's output are fine),
    ``key_cache`` and ``value_cache`` [pages, page_size, heads, dim] with any order of their first three
    dimensions, bfloat16 or float16.  ``slots`` (int64 [tokens]) are those of ``step_plan``; a token whose
    slot is not in the cache is passed over.  With ``frequencies`` (float32 [pairs]) and ``positions``
    (int32 [tokens]) the first 2 * pairs elements of each key are rotated on the way, as halves or as
    ``interleaved`` neighbours, and ``queries`` [tokens, q_heads, dim] into ``rotated`` (may be ``queries``).
    """
    cache, d = _cache(key_cache, value_cache)
    _, _, heads, dim = key_cache.shape
    dtype = key_cache.dtype
    k, k_stride = _heads(keys, "keys", d, dtype, None, heads, dim)
    n = keys.shape[0]
    v, v_stride = _heads(values, "values", d, dtype, n, heads, dim)
    if (queries is None) != (rotated is None):
        raise ValueError("queries and rotated come together")
    if queries is None:
        q_heads, q, q_stride, r, r_stride = 0, None, 0, None, 0
    else:
        q, q_stride = _heads(queries, "queries", d, dtype, n, None, dim)
        q_heads = queries.shape[1]
        r, r_stride = _heads(rotated, "rotated", d, dtype, n, q_heads, dim)
    pairs = 0
    if frequencies is not None:
        if positions is None:
            raise ValueError("frequencies need positions")
        pairs = _entries(frequencies, "frequencies")
    _lib.check(_lib.load().tt_cache_append(
        cache, n, _flat(slots, "slots", _I64, (n,), d), _flat(positions, "positions", _I32, (n,), d),
        _flat(frequencies, "frequencies", _F32, (pairs,), d), pairs, 1 if interleaved else 0, k, k_stride, v, v_stride,
        q_heads, q, q_stride, r, r_stride, stream), "tt_cache_append")


def cache_attention_workspace(tokens, requests, q_heads, kv_heads, dim) -> int:
    """``tt_cache_attention_workspace``: bytes of workspace that ``cache_attention`` needs."""
    return _need("tt_cache_attention_workspace", tokens, requests, q_heads, kv_heads, dim)


def cache_attention(queries, key_cache, value_cache, tables, offsets, lengths, out, logsums=None, scale=None, window=0, sinks=0,
                    workspace=None, stream=None):
    """``tt_cache_attention``: attention of a step's tokens over the paged cache of ``cache_append``.

    ``queries`` and ``out`` are [tokens, q_heads, dim]; ``tables``, ``offsets`` and ``lengths`` are those of
    ``step_plan`` (the tables with the step's pages).  A token sees its request's tokens up to itself, with
    ``window`` the last ``window`` of them and the first ``sinks``.  ``logsums`` (float32 [tokens, q_heads])
    receives the logarithms of the softmax's sums; ``scale`` is dim ** -0.5 by default.
    """
    cache, d = _cache(key_cache, value_cache)
    _, _, heads, dim = key_cache.shape
    dtype, n = key_cache.dtype, _entries(lengths, "lengths")
    q, q_stride = _heads(queries, "queries", d, dtype, None, None, dim)
    tokens, q_heads, _ = queries.shape
    o, o_stride = _heads(out, "out", d, dtype, tokens, q_heads, dim)
    table, t_stride = _matrix(tables, "tables", d)
    if _code(tables.dtype) != _I32 or tables.shape[0] != n:
        raise ValueError("tables must be an int32 matrix of %d rows, not %s %s" % (n, tables.dtype, tuple(tables.shape)))
    if not (0 <= window <= 0x7FFFFFFF and 0 <= sinks <= 0x7FFFFFFF):
        raise ValueError("window %r and sinks %r must be numbers of tokens below 2^31" % (window, sinks))
    if max(tokens, n, q_heads, tables.shape[1]) > 0x7FFFFFFF:
        raise ValueError("sizes past 32 bits")
    if heads < 1 or q_heads < 1 or q_heads % heads:
        raise ValueError("%d heads of queries are not a multiple of %d of keys" % (q_heads, heads))
    flat = _flat
    step = _ATTENTION.pack(
        n, tables.shape[1], t_stride, tokens, q_heads, window, sinks, dim ** -0.5 if scale is None else scale, q_stride,
        o_stride, table, flat(offsets, "offsets", _I32, (n + 1,), d), flat(lengths, "lengths", _I32, (n,), d), q, o,
        flat(logsums, "logsums", _F32, (tokens, q_heads), d))
    room, size = _room(workspace, _need("tt_cache_attention_workspace", tokens, n, q_heads, heads, dim), d)
    _lib.check(_lib.load().tt_cache_attention(cache, step, room, size, stream), "tt_cache_attention")


def _adjustment(logits, device, history, history_offsets, repetition, presence, frequency, bias_ids, bias_values, bias_offsets,
                masks, mask_rows):
    """tt_adjustment of these tensors."""
    p, stride = _matrix(logits, "logits", device)
    kind = _type_of(logits, "logits", (0, 1, 2))
    rows, vocab = logits.shape
    if (history is None) != (history_offsets is None) or (masks is None) != (mask_rows is None):
        raise ValueError("history and history_offsets, masks and mask_rows come together")
    if not (bias_ids is None) == (bias_values is None) == (bias_offsets is None):
        raise ValueError("bias_ids, bias_values and bias_offsets come together")
    if history is None and not (repetition is None and presence is None and frequency is None):
        raise ValueError("penalties need a history")
    n_history = n_biases = n_masks = mask = mask_stride = 0
    if history is not None:
        n_history = _entries(history, "history")
    if bias_ids is not None:
        n_biases = _entries(bias_ids, "bias_ids")
    if masks is not None:
        mask, mask_stride = _matrix(masks, "masks", device)
        n_masks, words = masks.shape
        if _code(masks.dtype) != _I32 or words < (vocab + 31) // 32 or n_masks > 0x7FFFFFFF:
            raise ValueError("masks must be an int32 matrix of at least %d words a row, not %s %s"
                             % ((vocab + 31) // 32, masks.dtype, tuple(masks.shape)))
    one, ends = (rows,), (rows + 1,)
    return _ADJUSTMENT.pack(
        kind, n_masks, rows, vocab, stride, n_history, n_biases, mask_stride, p,
        _flat(history, "history", _I32, (n_history,), device), _flat(history_offsets, "history_offsets", _I64, ends, device),
        _flat(repetition, "repetition", _F32, one, device), _flat(presence, "presence", _F32, one, device),
        _flat(frequency, "frequency", _F32, one, device), _flat(bias_ids, "bias_ids", _I32, (n_biases,), device),
        _flat(bias_values, "bias_values", _F32, (n_biases,), device), _flat(bias_offsets, "bias_offsets", _I64, ends, device),
        mask, _flat(mask_rows, "mask_rows", _I32, one, device))


def adjust_logits(logits, out, history=None, history_offsets=None, repetition=None, presence=None, frequency=None, bias_ids=None,
                  bias_values=None, bias_offsets=None, masks=None, mask_rows=None, stream=None):
    """``tt_adjust_logits``: penalties for repeated tokens, biases and masks on logits [rows, vocab].

    ``history`` (int32) holds the rows' tokens one row after the other, row r's between
    ``history_offsets[r]`` and ``[r + 1]`` (int64 [rows + 1]); ``repetition``, ``presence`` and
    ``frequency`` are float32 [rows].  ``bias_ids`` (int32) and ``bias_values`` (float32) are lists of the
    same kind with ``bias_offsets``.  ``masks`` (int32 [masks, words]) holds a bit a token, 1 where it is
    allowed, and ``mask_rows`` (int32 [rows]) each row's mask, negative for none.  ``out`` has the type
    and shape of the logits, and may be the logits.
    """
    d = _device(logits, "logits")
    a = _adjustment(logits, d, history, history_offsets, repetition, presence, frequency, bias_ids, bias_values, bias_offsets,
                    masks, mask_rows)
    _lib.check(_lib.load().tt_adjust_logits(a, *_matrix(out, "out", d, logits.dtype, logits.shape), stream), "tt_adjust_logits")


def adjust_logits_grad(logits, grad_out, grad_logits, history=None, history_offsets=None, repetition=None, masks=None,
                       mask_rows=None, stream=None):
    """``tt_adjust_logits_grad``: gradient with respect to the logits, into ``grad_logits`` (may be
    ``grad_out``), from that with respect to the adjusted logits; the other arguments are the call's."""
    d = _device(logits, "logits")
    a = _adjustment(logits, d, history, history_offsets, repetition, None, None, None, None, None, masks, mask_rows)
    _lib.check(_lib.load().tt_adjust_logits_grad(
        a, *_matrix(grad_out, "grad_out", d, logits.dtype, logits.shape),
        *_matrix(grad_logits, "grad_logits", d, logits.dtype, logits.shape), stream), "tt_adjust_logits_grad")


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
