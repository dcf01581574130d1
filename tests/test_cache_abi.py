"""The calls on a paged cache and on logits without a GPU: structures, and what they refuse before any device work."""

import ctypes
import os
import re

import pytest

import paper_2607_29678_amd as tt
from paper_2607_29678_amd import TokTierError, _lib, model

torch = pytest.importorskip("torch")
from test_model_device import Library, OnDevice  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, BAD, LARGE = 0, -1, -9, -6
P = 0x1000  # an address that is never followed
BF, I32, I64 = torch.bfloat16, torch.int32, torch.int64


@pytest.mark.parametrize("name,struct,packed", [("tt_cache", _lib.Cache, model._CACHE), ("tt_attention", _lib.Attention, model._ATTENTION),
                                                ("tt_adjustment", _lib.Adjustment, model._ADJUSTMENT)])
def test_structures_match_the_header(name, struct, packed):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "toktier_model.h")).read(), flags=re.S)
    body = [b for b, n in re.findall(r"typedef struct \{([^{}]*)\} (\w+);", src) if n == name][0]
    types = {"int32_t": _lib._I32, "int64_t": _lib._I64, "float": _lib._F}
    want = []
    for line in body.split(";"):
        m = re.match(r"\s*(?:const )?(\w+)(\*)? (.*)", line.strip())
        for field in m.group(3).split(",") if m else ():
            want.append((field.strip(), _lib._P if m.group(2) else types[m.group(1)]))
    assert [(n, t) for n, t in struct._fields_] == want
    assert packed.size == ctypes.sizeof(struct)
    values = list(range(1, len(want) + 1))
    s = struct.from_buffer_copy(packed.pack(*values))
    assert [getattr(s, n) for n, _ in struct._fields_] == values


def cache(**change):
    c = _lib.Cache(1, 16, 2, 64, 10, 16 * 128, 128, 64, P, 2 * P)
    for k, v in change.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [dict(type=0), dict(type=3), dict(page_size=0), dict(page_size=-1), dict(kv_heads=0), dict(dim=0), dict(dim=12),
              dict(dim=264), dict(pages=-1), dict(pages=1 << 31), dict(page_stride=-8), dict(slot_stride=4), dict(head_stride=1),
              dict(keys=P + 8), dict(values=P + 2)]


def _append(c=None, tokens=4, slots=P, positions=P, frequencies=P, pairs=32, inter=0, keys=P, ks=128, values=P, vs=128, qh=4,
            queries=P, qs=256, rotated=2 * P, rs=256):
    c = cache() if c is None else c
    return _lib.load().tt_cache_append(ctypes.byref(c), tokens, slots, positions, frequencies, pairs, inter, keys, ks, values, vs,
                                       qh, queries, qs, rotated, rs, None)


def _attention(c=None, work=P, size=1 << 40, **change):
    c = cache() if c is None else c
    s = _lib.Attention(3, 5, 5, 7, 4, 0, 0, 0.125, 256, 256, P, P, P, P, 2 * P, P)
    for k, v in change.items():
        setattr(s, k, v)
    return _lib.load().tt_cache_attention(ctypes.byref(c), ctypes.byref(s), work, size, None)


@pytest.mark.parametrize("change", BAD_CACHES)
def test_caches(change):
    assert _append(cache(**change)) == BAD
    assert _attention(cache(**change)) == BAD


def test_no_structures():
    lib = _lib.load()
    assert lib.tt_cache_append(None, 1, P, P, P, 1, 0, P, 128, P, 128, 0, None, 0, None, 0, None) == NULL
    s, c = _lib.Attention(), cache()
    assert lib.tt_cache_attention(None, ctypes.byref(s), P, 1 << 30, None) == NULL
    assert lib.tt_cache_attention(ctypes.byref(c), None, P, 1 << 30, None) == NULL
    assert lib.tt_adjust_logits(None, P, 100, None) == NULL
    assert lib.tt_adjust_logits_grad(None, P, 100, P, 100, None) == NULL


@pytest.mark.parametrize("change", [dict(tokens=-1), dict(tokens=1 << 31), dict(pairs=-1), dict(pairs=33), dict(ks=127), dict(vs=127),
                                    dict(qh=-1), dict(qs=255), dict(rs=255), dict(rotated=P, rs=264)])
def test_append_sizes(change):
    assert _append(**change) == BAD


def test_append_pointers():
    for name in ("slots", "positions", "frequencies", "keys", "values", "queries", "rotated"):
        assert _append(**{name: None}) == NULL, name
    assert _append(cache(keys=None)) == NULL
    assert _append(tokens=0, slots=None, keys=None) == OK
    assert _append(cache(kv_heads=200, dim=256), ks=1 << 20, vs=1 << 20, qs=1 << 20, rs=1 << 20) == LARGE


@pytest.mark.parametrize("change", [dict(n_requests=-1), dict(table_width=-1), dict(table_stride=4), dict(tokens=-1), dict(tokens=1 << 31),
                                    dict(q_heads=0), dict(q_heads=3), dict(window=-1), dict(sinks=-1), dict(scale=0.0),
                                    dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(query_stride=255),
                                    dict(out_stride=255), dict(out=P), dict(work=P + 128)])
def test_attention_sizes(change):
    assert _attention(**change) == BAD


def test_attention_pointers_and_workspace():
    for name in ("tables", "offsets", "lengths", "queries", "out"):
        assert _attention(**{name: None}) == NULL, name
    assert _attention(cache(values=None)) == NULL
    assert _attention(cache(page_stride=1 << 36)) == LARGE and _attention(cache(slot_stride=1 << 36)) == LARGE
    assert _attention(tokens=(1 << 31) - 1, n_requests=3) == LARGE
    assert _attention(tokens=0, queries=None, out=None) == OK
    assert _attention(n_requests=0, offsets=None) == OK
    need = tt.cache_attention_workspace(7, 3, 4, 2, 64)
    assert need >= 0
    if need:
        assert _attention(size=need - 1) == BAD
        assert _attention(work=None) == NULL
    for args in ((-1, 3, 4, 2, 64), (7, -1, 4, 2, 64), (7, 3, 0, 2, 64), (7, 3, 3, 2, 64), (7, 3, 4, 0, 64), (7, 3, 4, 2, 12),
                 (7, 3, 4, 2, 264)):
        with pytest.raises(TokTierError):
            tt.cache_attention_workspace(*args)


def _adjust(grad=False, out=2 * P, out_stride=100, go=3 * P, go_stride=100, **change):
    a = _lib.Adjustment(1, 2, 4, 100, 100, 10, 10, 4, *[P] * 11)
    for k, v in change.items():
        setattr(a, k, v)
    if grad:
        return _lib.load().tt_adjust_logits_grad(ctypes.byref(a), go, go_stride, out, out_stride, None)
    return _lib.load().tt_adjust_logits(ctypes.byref(a), out, out_stride, None)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("change", [dict(type=3), dict(type=-1), dict(n_masks=-1), dict(rows=-1), dict(vocab=0), dict(vocab=1 << 31),
                                    dict(stride=99), dict(n_history=-1), dict(n_biases=-1), dict(mask_stride=3), dict(history=None),
                                    dict(history_offsets=None), dict(bias_ids=None), dict(bias_values=None), dict(bias_offsets=None),
                                    dict(masks=None), dict(mask_rows=None), dict(out_stride=99)])
def test_adjustment_sizes(change, grad):
    assert _adjust(grad, **change) == BAD


def test_adjustment_pointers_and_places():
    assert _adjust(history=None, history_offsets=None, n_history=0) == BAD  # penalties without a history
    assert _adjust(out=None) == NULL
    assert _adjust(logits=None) == NULL
    assert _adjust(True, logits=None) == NULL
    assert _adjust(True, go=None) == NULL
    assert _adjust(True, out=None) == NULL
    assert _adjust(True, go_stride=99) == BAD
    assert _adjust(out=P, out_stride=108) == BAD
    assert _adjust(True, out=P) == BAD
    assert _adjust(True, go=2 * P, go_stride=108) == BAD
    assert _adjust(rows=0, out=None, logits=None) == OK
    assert _adjust(True, rows=0, go=None, out=None, logits=None) == OK
    assert _adjust(rows=1 << 40) == LARGE
    assert _adjust(n_history=1 << 32) == LARGE and _adjust(n_biases=1 << 32) == LARGE


# ---- the binding's own checks --------------------------------------------------------------------


@pytest.fixture
def library(monkeypatch):
    def use(current):
        lib = Library(current)
        monkeypatch.setattr(_lib, "load", lambda: lib)
        model._need.cache_clear()
        return lib

    yield use
    model._need.cache_clear()


def f(*s, t=torch.float32, device=0):
    return OnDevice(torch.zeros(s, dtype=t), device)


def calls(device):
    g = lambda *s, t=torch.float32: f(*s, t=t, device=device)  # noqa: E731
    return {
        "tt_cache_append": lambda: tt.cache_append(g(3, 2, 64, t=BF), g(3, 2, 64, t=BF), g(5, 16, 2, 64, t=BF), g(5, 16, 2, 64, t=BF),
                                                   g(3, t=I64), g(3, t=I32), g(32), False, g(3, 4, 64, t=BF), g(3, 4, 64, t=BF)),
        "tt_cache_attention": lambda: tt.cache_attention(g(3, 4, 64, t=BF), g(5, 16, 2, 64, t=BF), g(5, 16, 2, 64, t=BF),
                                                         g(2, 7, t=I32), g(3, t=I32), g(2, t=I32), g(3, 4, 64, t=BF), g(3, 4)),
        "tt_adjust_logits": lambda: tt.adjust_logits(g(3, 100), g(3, 100), g(9, t=I32), g(4, t=I64), g(3), g(3), g(3), g(5, t=I32),
                                                     g(5), g(4, t=I64), g(2, 4, t=I32), g(3, t=I32)),
        "tt_adjust_logits_grad": lambda: tt.adjust_logits_grad(g(3, 100), g(3, 100), g(3, 100), g(9, t=I32), g(4, t=I64), g(3),
                                                               g(2, 4, t=I32), g(3, t=I32)),
    }


@pytest.mark.parametrize("name", sorted(calls(0)))
def test_the_device_has_to_be_the_current_one(library, name):
    for current, device in ((0, 1), (1, 0), (-7, 0)):
        lib = library(current)
        with pytest.raises(ValueError):
            calls(device)[name]()
        assert lib.calls == []
    for device in (0, 1):
        lib = library(device)
        calls(device)[name]()
        assert lib.calls == [name]
    for name in calls(-1):
        with pytest.raises(ValueError):
            calls(-1)[name]()


def refused(lib, call, good, changes):
    call(**good)
    n = len(lib.calls)
    for change in changes:
        with pytest.raises(ValueError):
            call(**{**good, **change})
    assert len(lib.calls) == n


def test_append_arguments(library):
    good = dict(keys=f(3, 2, 64, t=BF), values=f(3, 2, 64, t=BF), key_cache=f(5, 16, 2, 64, t=BF), value_cache=f(5, 16, 2, 64, t=BF),
                slots=f(3, t=I64), positions=f(3, t=I32), frequencies=f(32), queries=f(3, 4, 64, t=BF), rotated=f(3, 4, 64, t=BF))
    wide = torch.zeros(3, 4, 64, dtype=BF)
    refused(library(0), tt.cache_append, good, [
        dict(keys=f(3, 2, 64)), dict(keys=f(4, 2, 64, t=BF)), dict(keys=f(3, 1, 64, t=BF)), dict(keys=f(3, 2, 32, t=BF)),
        dict(keys=f(3, 128, t=BF)), dict(keys=OnDevice(wide[:, ::2], 0)), dict(values=OnDevice(wide[:1, :2].expand(3, 2, 64), 0)),
        dict(values=OnDevice(torch.zeros(3, 64, 2, dtype=BF).transpose(1, 2), 0)), dict(values=f(3, 2, 64, t=BF, device=1)),
        dict(key_cache=f(5, 16, 2, 64)), dict(value_cache=f(5, 16, 2, 32, t=BF)), dict(value_cache=f(5, 16, 2, 64, t=torch.float16)),
        dict(key_cache=OnDevice(torch.zeros(16, 5, 2, 64, dtype=BF).transpose(0, 1), 0)),
        dict(key_cache=OnDevice(torch.zeros(1, 16, 2, 64, dtype=BF).expand(5, 16, 2, 64), 0),
             value_cache=OnDevice(torch.zeros(1, 16, 2, 64, dtype=BF).expand(5, 16, 2, 64), 0)),
        dict(slots=f(3, t=I32)), dict(slots=f(2, t=I64)), dict(positions=None), dict(positions=f(3, t=I64)), dict(frequencies=f(32, t=BF)),
        dict(frequencies=f(2, 32)), dict(rotated=None), dict(queries=None), dict(rotated=f(3, 2, 64, t=BF)), dict(queries=f(4, 4, 64, t=BF))])


def test_attention_arguments(library):
    good = dict(queries=f(3, 4, 64, t=BF), key_cache=f(5, 16, 2, 64, t=BF), value_cache=f(5, 16, 2, 64, t=BF), tables=f(2, 7, t=I32),
                offsets=f(3, t=I32), lengths=f(2, t=I32), out=f(3, 4, 64, t=BF), logsums=f(3, 4))
    refused(library(0), tt.cache_attention, good, [
        dict(queries=f(3, 4, 64)), dict(queries=f(3, 3, 64, t=BF)), dict(queries=f(3, 4, 32, t=BF)), dict(out=f(3, 4, 64)),
        dict(out=f(2, 4, 64, t=BF)), dict(tables=f(3, 7, t=I32)), dict(tables=f(2, 7, t=I64)), dict(tables=f(14, t=I32)),
        dict(offsets=f(2, t=I32)), dict(offsets=f(3, t=I64)), dict(lengths=f(2, t=I64)), dict(logsums=f(4, 3)), dict(logsums=f(3, 4, t=BF)),
        dict(window=-1), dict(sinks=-1), dict(window=1 << 31), dict(sinks=1 << 31)])


def test_adjustment_arguments(library):
    good = dict(logits=f(3, 100), out=f(3, 100), history=f(9, t=I32), history_offsets=f(4, t=I64), repetition=f(3), presence=f(3),
                frequency=f(3), bias_ids=f(5, t=I32), bias_values=f(5), bias_offsets=f(4, t=I64), masks=f(2, 4, t=I32),
                mask_rows=f(3, t=I32))
    refused(library(0), tt.adjust_logits, good, [
        dict(logits=f(3, 100, t=torch.float64)), dict(out=f(3, 100, t=BF)), dict(out=f(3, 99)), dict(history=f(9, t=I64)),
        dict(history=None), dict(history_offsets=None), dict(history_offsets=f(3, t=I64)), dict(history_offsets=f(4, t=I32)),
        dict(history=None, history_offsets=None), dict(repetition=f(4)), dict(presence=f(3, t=BF)), dict(bias_ids=None),
        dict(bias_values=f(4)), dict(bias_values=None), dict(bias_offsets=None), dict(bias_offsets=f(5, t=I64)), dict(masks=None),
        dict(mask_rows=None), dict(masks=f(2, 3, t=I32)), dict(masks=f(2, 4)), dict(mask_rows=f(2, t=I32))])
    good = {k: v for k, v in good.items() if k in ("logits", "history", "history_offsets", "repetition", "masks", "mask_rows")}
    good.update(grad_out=f(3, 100), grad_logits=f(3, 100))
    refused(library(0), tt.adjust_logits_grad, good, [
        dict(grad_out=f(3, 99)), dict(grad_logits=f(3, 100, t=BF)), dict(history=None), dict(repetition=f(2)), dict(masks=None)])
