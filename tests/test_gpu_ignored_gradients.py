"""Head gradients beside values that belong to no token: what stands at a row that the call ignores changes no other row.

The 16-bit floats of G are scaled by one power of two, taken from the gradients that count: those of rows with a given
token and a distribution.
"""

import math

import pytest

torch = pytest.importorskip("torch")
import paper_2607_29678_amd as tt  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]
VOCAB, WIDTH = 1_281, 128


def make(rows, kind, seed=5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    weight = (torch.randn(VOCAB, WIDTH, generator=gen, device="cuda") * WIDTH**-0.5).to(kind)
    hidden = torch.randn(rows, WIDTH, generator=gen, device="cuda").to(kind)
    targets = torch.randint(0, VOCAB, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    g = (torch.rand(rows, generator=gen, device="cuda") + 0.5) / rows
    return hidden, weight, targets, g


def gradients(hidden, weight, targets, g, ge=None):
    rows = len(hidden)
    z = hidden.double() @ weight.double().t().contiguous()
    m = z.amax(1)
    stats = torch.stack([m, (z - m[:, None]).exp().sum(1).log()], 1).float()
    lp = z.log_softmax(1)
    entropy = -(lp.exp() * lp).sum(1).float()
    room = torch.empty(tt.head_scores_grad_workspace(rows, VOCAB, WIDTH), dtype=torch.uint8, device="cuda")
    gh, gw = torch.full_like(hidden, 55.0), torch.full_like(weight, 55.0)
    tt.head_scores_grad(hidden, weight, targets, stats, entropy, g, ge, gh, gw, workspace=room)
    torch.cuda.synchronize()
    return gh, gw


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [3, 200, 300])
@pytest.mark.parametrize("value", [1e30, -1e30, math.inf, -math.inf, math.nan])
def test_gradient_where_no_token_is_given(gpu, rows, kind, value):
    hidden, weight, targets, g = make(rows, kind)
    targets[1::3] = -1
    g[1::3] = 0.0
    want = gradients(hidden, weight, targets, g)
    assert float(want[0].float().abs().sum()) > 0
    g[1::3] = value
    got = gradients(hidden, weight, targets, g)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("rows", [3, 300])
def test_gradients_of_no_tokens_at_all(gpu, rows):
    """Without targets only the entropies pass a gradient on."""
    hidden, weight, _, g = make(rows, torch.float16)
    want = gradients(hidden, weight, None, None, g)
    got = gradients(hidden, weight, None, torch.full_like(g, 1e30), g)
    assert float(want[0].float().abs().sum()) > 0
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("how", ["past", "infinite", "nan"])
def test_a_row_without_numbers_spoils_no_other(gpu, rows, how):
    """A row whose own gradient is no number (a target past the vocabulary, a gradient that is infinite or NaN): the
    other rows' hidden gradients are those beside a row of zeros."""
    hidden, weight, targets, g = make(rows, torch.float16)
    g[1] = 0.0
    want, _ = gradients(hidden, weight, targets, g)
    if how == "past":
        targets[1], g[1] = VOCAB, 1e30
    else:
        g[1] = math.inf if how == "infinite" else math.nan
    got, _ = gradients(hidden, weight, targets, g)
    others = torch.arange(rows, device="cuda") != 1
    assert torch.equal(got[others], want[others])
    assert not bool(torch.isfinite(got[1]).any())
