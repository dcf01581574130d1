"""``toktier_model.h`` without a GPU: exports, declarations, and what the calls refuse before any device work."""

import ctypes
import os
import re

import pytest

from paper_2607_29678_amd import (TokTierError, _lib, head_scores, head_scores_grad, head_scores_grad_workspace,
                                  head_scores_workspace, step_plan, token_scores, token_scores_grad,
                                  token_scores_workspace)

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, BAD, LARGE = -1, -9, -6
P = 0x1000  # an address that is never followed


def _header():
    src = open(os.path.join(ROOT, "include", "toktier_model.h")).read()
    return re.sub(r"/\*.*?\*/", "", src, flags=re.S)


def test_declared_and_exported():
    names = sorted(set(re.findall(r"\b(tt_[a-z_]+)\s*\(", _header())))
    assert names == sorted(_lib.MODEL_SIGNATURES)
    lib = _lib.load()
    for n in names:
        assert hasattr(lib, n), n


def test_step_matches_the_header():
    body = re.search(r"typedef struct \{(.*?)\} tt_step;", _header(), flags=re.S).group(1)
    fields = re.findall(r"(\w+)\s*(\*)?\s*(\w+);", body)
    want = [(n, _lib._P if star else {"int32_t": _lib._I32, "int64_t": _lib._I64}[t]) for t, star, n in fields]
    assert [(n, t) for n, t in _lib.Step._fields_] == want


def test_packed_step_is_the_struct():
    from paper_2607_29678_amd import model

    values = list(range(1, 22))
    step = _lib.Step.from_buffer_copy(model._STEP.pack(*values))
    assert [getattr(step, n) for n, _ in _lib.Step._fields_] == values


def _step(**change):
    s = _lib.Step(4, 16, 10, 10, 64, 100, *range(P, P + 15 * 64, 64))
    for k, v in change.items():
        setattr(s, k, v)
    return _lib.load().tt_step_plan(ctypes.byref(s), None)


@pytest.mark.parametrize("change", [dict(n_requests=-1), dict(page_size=0), dict(page_size=-16), dict(table_width=-1),
                                    dict(table_stride=9), dict(max_tokens=-1), dict(max_tokens=1 << 31), dict(n_free=-1),
                                    dict(n_free=1 << 31), dict(ids=None), dict(targets=None)])
def test_step_sizes(change):
    assert _step(**change) == BAD


@pytest.mark.parametrize("name", ["cached", "fresh", "free_pages", "free_count", "tables", "offsets", "lengths", "pages",
                                  "slots", "positions", "requests", "result"])
def test_step_pointers(name):
    assert _step(**{name: None}) == NULL
    assert _lib.load().tt_step_plan(None, None) == NULL


@pytest.mark.parametrize("out,inp", [("result", "free_count"), ("pages", "held"), ("lengths", "cached"),
                                     ("lengths", "fresh"), ("targets", "ids")])
def test_step_outputs_are_not_inputs(out, inp):
    assert _step(**{out: 0x9000, inp: 0x9000}) == BAD
    if out == "result":
        assert _step(result=0x9000, free_count=0x9008) == BAD


def _scores(rows=4, vocab=100, stride=100, kind=1, scale=1.0, n_alt=0, logits=P, ai=P, al=P, work=P, size=1 << 20):
    return _lib.load().tt_token_scores(logits, kind, rows, vocab, stride, scale, P, P, P, P, n_alt, ai, al, work, size, None)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(vocab=0), dict(vocab=1 << 31, stride=1 << 31), dict(stride=99),
                                    dict(kind=3), dict(kind=-1), dict(scale=0.0), dict(scale=-1.0),
                                    dict(scale=float("inf")), dict(scale=float("nan")), dict(n_alt=-1), dict(n_alt=65),
                                    dict(vocab=50_000, stride=50_000, size=100)])
def test_scores_sizes(change):
    assert _scores(**change) == BAD


def test_scores_pointers():
    assert _scores(logits=None) == NULL
    assert _scores(n_alt=3, ai=None) == NULL
    assert _scores(n_alt=3, al=None) == NULL
    assert _scores(vocab=50_000, stride=50_000, work=None) == NULL
    assert _scores(rows=1 << 40) == LARGE
    assert _scores(rows=0, logits=None, work=None, size=0) == 0


def _grad(rows=4, vocab=100, stride=100, kind=1, scale=1.0, logits=P, stats=P, entropy=P, ge=P, out=2 * P, out_stride=100):
    return _lib.load().tt_token_scores_grad(logits, kind, rows, vocab, stride, scale, P, stats, entropy, P, ge, out,
                                            out_stride, None)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(vocab=0), dict(stride=99), dict(out_stride=99), dict(kind=5),
                                    dict(scale=0.0), dict(out=P, out_stride=200)])
def test_grad_sizes(change):
    assert _grad(**change) == BAD


def test_grad_pointers():
    assert _grad(logits=None) == NULL
    assert _grad(out=None) == NULL
    assert _grad(stats=None) == NULL
    assert _grad(entropy=None) == NULL
    assert _grad(rows=0, logits=None, out=None) == 0
    assert _grad(rows=1 << 40) == LARGE


def _head(rows=4, vocab=100, width=64, hs=64, ws=64, kind=1, scale=1.0, hidden=P, weight=P, work=P, size=1 << 20):
    return _lib.load().tt_head_scores(hidden, hs, weight, ws, kind, rows, vocab, width, scale, P, P, P, P, work, size, None)


def _head_grad(rows=4, vocab=100, width=64, hs=64, ws=64, kind=1, scale=1.0, hidden=P, weight=P, stats=P, entropy=P, ge=P,
               gh=P, ghs=64, gw=P, gws=64, work=P, size=1 << 24):
    return _lib.load().tt_head_scores_grad(hidden, hs, weight, ws, kind, rows, vocab, width, scale, P, stats, entropy, P, ge,
                                           gh, ghs, gw, gws, work, size, None)


@pytest.mark.parametrize("call", [_head, _head_grad])
@pytest.mark.parametrize("change", [dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(width=0),
                                    dict(hs=63), dict(ws=63), dict(kind=0), dict(kind=3), dict(scale=0.0), dict(size=10)])
def test_head_sizes(call, change):
    assert call(**change) == BAD


def test_head_grad_strides_and_pointers():
    assert _head_grad(ghs=63) == BAD
    assert _head_grad(gws=63) == BAD
    for name in ("hidden", "weight", "stats", "entropy", "work"):
        assert _head_grad(**{name: None}) == NULL
    assert _head_grad(gh=None, gw=None) == 0
    for name in ("hidden", "weight", "work"):
        assert _head(**{name: None}) == NULL
    assert _head(rows=0, hidden=None, work=None, size=0) == 0


def test_workspace_alignment():
    assert _scores(vocab=50_000, stride=50_000, work=P + 8) == BAD
    assert _head(work=P + 128) == BAD
    assert _head_grad(work=P + 16) == BAD


def test_widths_past_a_buffer():
    lib = _lib.load()
    assert lib.tt_head_scores_grad_workspace(8, 100, (1 << 21) + 1, 1) == LARGE
    assert _head_grad(width=(1 << 21) + 8, hs=1 << 22, ws=1 << 22, ghs=1 << 22, gws=1 << 22, size=1 << 62) == LARGE


def test_workspaces():
    assert token_scores_workspace(5000, 100_257, 20) == 0
    assert token_scores_workspace(1, 100_257, 20) > 0
    assert head_scores_workspace(0, 100, 64) == 0
    for args in ((-1, 5, 0), (5, 0, 0), (5, 5, 65)):
        with pytest.raises(TokTierError):
            token_scores_workspace(*args)
    with pytest.raises(TokTierError):
        head_scores_workspace(5, 5, 0)
    for rows, vocab, width in ((1, 1, 1), (640, 50_257, 1024), (4001, 100_257, 2048)):
        assert 0 < head_scores_grad_workspace(rows, vocab, width, False) <= head_scores_grad_workspace(rows, vocab, width, True)


# ---- the binding's own checks (CPU tensors never get past them) ----


def test_binding_refuses_host_tensors():
    f, i = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    z = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        token_scores(z, i, f)
    with pytest.raises(ValueError):
        token_scores_grad(z, i, torch.zeros(4, 2), f, f, f, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        head_scores(z.half(), z.half(), i, f)
    with pytest.raises(ValueError):
        head_scores_grad(z.half(), z.half(), i, torch.zeros(4, 2), f, f, f, z.half(), z.half())
    with pytest.raises(ValueError):
        step_plan(i, i, z.int(), i, torch.zeros(1, dtype=torch.int64), 16, torch.zeros(5).int(), i, i,
                  torch.zeros(4, dtype=torch.int64), i, i, torch.zeros(2, dtype=torch.int64))
