"""What the binding of ``toktier_model.h`` refuses for device tensors: types, shapes, strides, workspaces."""

import pytest

torch = pytest.importorskip("torch")
from paper_2607_29678_amd import TokTierError, head_scores, head_scores_grad, step_plan, token_scores, token_scores_grad  # noqa: E402

pytestmark = pytest.mark.gpu


def f(*s, t=torch.float32):
    return torch.zeros(s, dtype=t, device="cuda")


I32, I64, U8 = torch.int32, torch.int64, torch.uint8


def test_scores(gpu):
    z, t, o, w = f(4, 5000), f(4, t=I32), f(4), f(1 << 16, t=U8)
    good = dict(logits=z, targets=t, logprobs=o, workspace=w)
    token_scores(**good)
    for change in (dict(logits=f(4, 5000, t=torch.float64)), dict(logits=f(5000)), dict(logits=f(5000, 4).t()),
                   dict(logits=f(1, 5000).expand(4, 5000)), dict(targets=f(4, t=I64)), dict(targets=f(5, t=I32)),
                   dict(logprobs=f(4, t=torch.float16)), dict(logprobs=f(8)[::2]), dict(stats=f(4)), dict(entropy=f(3)),
                   dict(alt_ids=f(4, 3, t=I32)), dict(alt_ids=f(4, 3, t=I32), alt_logprobs=f(4, 2)),
                   dict(workspace=None), dict(workspace=w[:16]), dict(workspace=w[8:]), dict(workspace=w.cpu()),
                   dict(targets=t.cpu())):
        with pytest.raises(ValueError):
            token_scores(**{**good, **change})
    with pytest.raises(TokTierError):
        token_scores(**good, scale=0.0)
    with pytest.raises(TokTierError):
        token_scores(**good, alt_ids=f(4, 65, t=I32), alt_logprobs=f(4, 65))
    torch.cuda.synchronize()


def test_scores_grad(gpu):
    z = f(4, 50)
    good = dict(logits=z, targets=f(4, t=I32), stats=f(4, 2), entropy=f(4), grad_logprobs=f(4), grad_entropy=f(4), grad_logits=f(4, 50))
    token_scores_grad(**good)
    for change in (dict(grad_logits=f(4, 50, t=torch.float16)), dict(grad_logits=f(4, 49)), dict(grad_logits=f(50, 4).t()),
                   dict(stats=f(4)), dict(grad_logprobs=f(4, 1)), dict(grad_entropy=f(5)), dict(entropy=f(4, t=torch.float64))):
        with pytest.raises(ValueError):
            token_scores_grad(**{**good, **change})
    for change in (dict(entropy=None), dict(stats=None)):
        with pytest.raises(TokTierError):
            token_scores_grad(**{**good, **change})
    torch.cuda.synchronize()


def test_head(gpu):
    h, w, room = f(4, 64, t=torch.bfloat16), f(90, 64, t=torch.bfloat16), f(1 << 22, t=U8)
    good = dict(hidden=h, weight=w, targets=f(4, t=I32), logprobs=f(4), workspace=room)
    head_scores(**good)
    for change in (dict(hidden=f(4, 64)), dict(hidden=h.half()), dict(weight=f(90, 63, t=torch.bfloat16)),
                   dict(hidden=f(4, 64), weight=f(90, 64)), dict(targets=f(3, t=I32)), dict(workspace=None),
                   dict(workspace=room[:8])):
        with pytest.raises(ValueError):
            head_scores(**{**good, **change})
    good = dict(hidden=h, weight=w, targets=f(4, t=I32), stats=f(4, 2), entropy=f(4), grad_logprobs=f(4), grad_entropy=f(4),
                grad_hidden=f(4, 64, t=torch.bfloat16), grad_weight=f(90, 64, t=torch.bfloat16), workspace=room)
    head_scores_grad(**good)
    for change in (dict(grad_hidden=f(4, 64)), dict(grad_hidden=f(4, 63, t=torch.bfloat16)),
                   dict(grad_weight=f(91, 64, t=torch.bfloat16)), dict(workspace=room[:256]), dict(stats=f(4))):
        with pytest.raises(ValueError):
            head_scores_grad(**{**good, **change})
    torch.cuda.synchronize()


def test_plan(gpu):
    n, room = 3, 8
    good = dict(cached=f(n, t=I32), fresh=f(n, t=I32), tables=f(n, 5, t=I32), free_pages=f(9, t=I32), free_count=f(1, t=I64),
                page_size=16, offsets=f(n + 1, t=I32), lengths=f(n, t=I32), pages=f(n, t=I32), slots=f(room, t=I64),
                positions=f(room, t=I32), requests=f(room, t=I32), result=f(2, t=I64), ids=f(room, t=I32), targets=f(room, t=I32))
    step_plan(**good)
    for change in (dict(cached=f(n, t=I64)), dict(fresh=f(n + 1, t=I32)), dict(tables=f(n + 1, 5, t=I32)),
                   dict(tables=f(n, 5)), dict(tables=f(5, n, t=I32).t()), dict(free_count=f(2, t=I64)),
                   dict(free_count=f(1, t=I32)), dict(offsets=f(n, t=I32)), dict(slots=f(room, t=I32)),
                   dict(positions=f(room - 1, t=I32)), dict(result=f(3, t=I64)), dict(held=f(n, t=I64)),
                   dict(ids=f(room + 1, t=I32)), dict(free_pages=f(18, t=I32)[::2]), dict(fresh=torch.zeros(n, dtype=I32))):
        with pytest.raises(ValueError):
            step_plan(**{**good, **change})
    for change in (dict(page_size=0), dict(targets=None), dict(ids=None), dict(lengths=good["cached"])):
        with pytest.raises(TokTierError):
            step_plan(**{**good, **change})
    torch.cuda.synchronize()
