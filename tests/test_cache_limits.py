"""The sizes that the calls on a paged cache and on logits refuse as too large, where the header says they are (CPU)."""

import pytest

import paper_2607_29678_amd as tt
from paper_2607_29678_amd import _lib, model

torch = pytest.importorskip("torch")
from test_cache_abi import LARGE, OK, _adjust, _append, cache, f  # noqa: E402
from test_model_device import Library  # noqa: E402


def append(q_heads, kv_heads, dim, tokens=0):
    c = cache(kv_heads=kv_heads, dim=dim, page_stride=16 * kv_heads * dim, slot_stride=kv_heads * dim, head_stride=dim)
    width = kv_heads * dim
    return _append(c, tokens=tokens, pairs=0, ks=width, vs=width, qh=q_heads, qs=q_heads * dim, rs=q_heads * dim)


@pytest.mark.parametrize("q_heads,kv_heads,dim", [(128, 64, 256), (128, 128, 192), (0, 128, 256), (8_190, 1, 8)])
def test_elements_of_a_token(q_heads, kv_heads, dim):
    assert (q_heads + 2 * kv_heads) * dim >= 65_536
    assert append(q_heads, kv_heads, dim) == LARGE
    q_heads, kv_heads = (q_heads - 1, kv_heads) if q_heads else (0, kv_heads - 1)
    if (q_heads + 2 * kv_heads) * dim <= 65_535:
        assert append(q_heads, kv_heads, dim) == OK


def test_tokens_of_an_append():
    # (refused before the launch: three tokens a block at most)
    assert append(4, 2, 64, tokens=3 * (1 << 24)) == LARGE


def test_columns_of_a_step():
    assert _adjust(vocab=4_096, stride=4_096, mask_stride=128, out_stride=4_096, rows=1 << 24) == LARGE
    assert _adjust(True, vocab=100_000, stride=100_000, mask_stride=3_125, out_stride=100_000, go_stride=100_000, rows=1 << 21) == LARGE
    assert _adjust(n_history=(1 << 32) - 1) == LARGE and _adjust(n_biases=(1 << 32) - 1) == LARGE


def test_a_workspace_of_any_lengths():
    for heads, kv, dim, most in ((32, 8, 128, 69e6), (16, 16, 64, 35e6), (3, 1, 256, 69e6)):
        sizes = {tt.cache_attention_workspace(tokens, requests, heads, kv, dim) for tokens in (1, 7, 100_000) for requests in (1, 3, 5_000)}
        assert len(sizes) == 1 and max(sizes) < most


def test_tensors_without_dimensions(monkeypatch):
    """A mismatch of shapes raises ValueError, whichever it is."""
    lib = Library(0)
    monkeypatch.setattr(_lib, "load", lambda: lib)
    model._need.cache_clear()
    B, I, L = torch.bfloat16, torch.int32, torch.int64
    caches = dict(key_cache=f(5, 16, 2, 64, t=B), value_cache=f(5, 16, 2, 64, t=B))
    good = [
        (tt.cache_append, dict(keys=f(3, 2, 64, t=B), values=f(3, 2, 64, t=B), slots=f(3, t=L), positions=f(3, t=I), frequencies=f(32),
                               queries=f(3, 4, 64, t=B), rotated=f(3, 4, 64, t=B), **caches)),
        (tt.cache_attention, dict(queries=f(3, 4, 64, t=B), tables=f(2, 7, t=I), offsets=f(3, t=I), lengths=f(2, t=I),
                                  out=f(3, 4, 64, t=B), logsums=f(3, 4), **caches)),
        (tt.adjust_logits, dict(logits=f(3, 100), out=f(3, 100), history=f(9, t=I), history_offsets=f(4, t=L), repetition=f(3),
                                bias_ids=f(5, t=I), bias_values=f(5), bias_offsets=f(4, t=L), masks=f(2, 4, t=I), mask_rows=f(3, t=I)))]
    for call, args in good:
        call(**args)
        n = len(lib.calls)
        for name, tensor in args.items():
            for shape in ((), (1,) * 5):
                with pytest.raises(ValueError):
                    call(**{**args, name: f(*shape, t=tensor.dtype)})
        assert len(lib.calls) == n
    model._need.cache_clear()
