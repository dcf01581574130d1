"""Rows that are nearly sure of one token: the scores, and the gradients from the scores' own statistics.

1 - p of such a token is the sum of all the others' exponentials, next to a 1 that would swallow its low bits.  All
bounds here are relative to the small values themselves.
"""

import math

import pytest

torch = pytest.importorskip("torch")
import model_reference as ref  # noqa: E402
import paper_2607_29678_amd as tt  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF = math.inf


def exact(z, scale=1.0):
    """log s, entropy and log probabilities of float64 logits, the largest entry apart from the others."""
    m, at = z.max(1, keepdim=True)
    d = (z - m) * scale
    others = torch.where(torch.arange(z.shape[1], device=z.device) == at, torch.zeros_like(d), d.exp())
    s = others.sum(1)
    log_s = torch.log1p(s)
    entropy = log_s - torch.where(others > 0, others * d, torch.zeros_like(d)).sum(1) / (1 + s)
    return dict(m=m[:, 0], log_s=log_s, entropy=entropy, lp=d - log_s[:, None], depth=float(torch.where(others > 0, -d, 0.0).max()))


def exact_grad(e, targets, a, b, scale=1.0):
    """(gradient with respect to the logits, sum of the sizes of its terms: those of 1 - p apart from p)."""
    p, lp = e["lp"].exp(), e["lp"]
    lp0 = torch.where(p > 0, lp, torch.zeros_like(lp))
    rows, t = torch.arange(len(p), device=p.device), targets.clamp(min=0).long()
    a = torch.where(targets < 0, torch.zeros_like(a), a)
    given = -p * a[:, None]
    given[rows, t] = torch.where(targets < 0, given[rows, t], -a * torch.expm1(lp[rows, t]))
    h = e["entropy"][:, None]
    g = scale * (given - b[:, None] * p * (lp0 + h))
    return g, scale * (given.abs() + b.abs()[:, None] * p * (lp0.abs() + h))


def relative_error(depth, vocab):
    """Of a sum of exponentials and of what is made of it: exponents up to `depth` with four roundings, the functions'
    own units, a lane's sum of vocab / 64 entries and the tree above it."""
    return ref.U32 * (4 * depth + 48 + vocab / 64)


def near(got, want, tol):
    ref.close(got, want, tol)


def scores_of(z, t, n_alt, scale):
    rows, vocab = z.shape
    f = lambda *s: torch.full(s, 77.0, device="cuda")  # noqa: E731
    out = dict(logprobs=f(rows), stats=f(rows, 2), entropy=f(rows))
    if n_alt:
        out.update(alt_ids=torch.full((rows, n_alt), -77, dtype=torch.int32, device="cuda"), alt_logprobs=f(rows, n_alt))
    work = torch.full((max(1, tt.token_scores_workspace(rows, vocab, n_alt)),), 255, dtype=torch.uint8, device="cuda")
    tt.token_scores(z, t, scale=scale, workspace=work, **out)
    torch.cuda.synchronize()
    return out


def sure_logits(rows, vocab, kind, lift, seed=3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, vocab, generator=gen, device="cuda") * 2.0).clamp(max=8.0)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    x[torch.arange(rows, device="cuda"), t.long()] = lift
    return x.to(kind), t


# rows of a block, of a wave and of several blocks
SHAPES = [(3, 1_281), (2_100, 1_281), (2_050, 16_384), (8, 50_257), (40, 8_449)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lift,scale", [(4.0, 1.0), (18.0, 1.0), (22.0, 1.0), (9.5, 2.0), (40.0, 0.5)])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_scores_of_sure_rows(gpu, rows, vocab, kind, lift, scale):
    z, t = sure_logits(rows, vocab, kind, lift)
    e = exact(z.double(), scale)
    tol = relative_error(e["depth"], vocab)
    want = e["lp"].gather(1, t.long()[:, None])[:, 0]
    for n_alt in (0, 5):
        got = scores_of(z, t, n_alt, scale)
        near(got["stats"][:, 1], e["log_s"], tol * e["log_s"])
        near(got["logprobs"], want, tol * want.abs())
        near(got["entropy"], e["entropy"], 2 * tol * e["entropy"])
        if n_alt:
            # (a lift of 4 does not reach over all the others)
            assert lift == 4.0 or torch.equal(got["alt_ids"][:, 0], t)
            near(got["alt_logprobs"][:, 0], e["lp"].amax(1), tol * e["lp"].amax(1).abs())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("entropy_weight", [0.0, 0.25])
@pytest.mark.parametrize("lift", [4.0, 18.0, 22.0])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_gradient_from_the_scores_own_statistics(gpu, rows, vocab, kind, lift, entropy_weight):
    z, t = sure_logits(rows, vocab, kind, lift)
    t[1::5] = -1
    e = exact(z.double())
    a = torch.linspace(0.7, 1.3, rows, device="cuda")
    b = torch.full((rows,), entropy_weight, device="cuda")
    s = scores_of(z, t, 0, 1.0)
    g = torch.full_like(z, 55.0)
    tt.token_scores_grad(z, t, s["stats"], s["entropy"], a, b, g)
    torch.cuda.synchronize()
    want, size = exact_grad(e, t, a.double(), b.double())
    unit, least = ref.ROUNDING[kind]
    near(g, want, size * (3 * relative_error(e["depth"], vocab) + 16 * ref.U32) + unit * want.abs() + least + 1e-37)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_rows_of_one_or_two_tokens(gpu, rows, vocab, kind):
    """One token left: nothing is uncertain.  Two equal ones: one bit."""
    z, t = sure_logits(rows, vocab, kind, 3.0)
    one = torch.full_like(z, -INF)
    one[torch.arange(rows, device="cuda"), t.long()] = 3.0
    for n_alt in (0, 3):
        got = scores_of(one, t, n_alt, 1.0)
        assert bool((got["stats"][:, 0] == 3).all()) and bool((got["stats"][:, 1] == 0).all())
        assert bool((got["logprobs"] == 0).all()) and bool((got["entropy"] == 0).all())
        two = one.clone()
        two[torch.arange(rows, device="cuda"), (t.long() + vocab // 3) % vocab] = 3.0
        got = scores_of(two, t, n_alt, 1.0)
        assert float((got["stats"][:, 1] - math.log(2)).abs().max()) <= 2e-7
        assert float((got["logprobs"] + math.log(2)).abs().max()) <= 2e-7
        assert float((got["entropy"] - math.log(2)).abs().max()) <= 2e-7


def sure_head(rows, vocab, width, kind, lift, seed=4):
    """Hidden states that point at one row of the weights, with a little noise."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    weight = torch.randn(vocab, width, generator=gen, device="cuda").to(kind)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    w = weight[t.long()].float()
    hidden = lift * w / (w * w).sum(1, keepdim=True) + 0.02 * torch.randn(rows, width, generator=gen, device="cuda")
    return hidden.to(kind), weight, t


HEADS = [(3, 1_281, 256), (40, 2_049, 512), (64, 700, 250), (100, 1_281, 256), (200, 1_500, 333), (300, 1_281, 256)]


def head_scores(hidden, weight, t):
    """(float64 logits, bound of a recomputed logit's error, their exact scores, the call's scores, scratch memory)."""
    rows, vocab, width = len(hidden), len(weight), hidden.shape[1]
    h, w = hidden.double(), weight.double()
    z = h @ w.t().contiguous()
    # `width` products summed in 32 bits, in any order
    off = float((h.abs() @ w.t().contiguous().abs()).max()) * width * ref.U32
    f = lambda *s: torch.full(s, 77.0, device="cuda")  # noqa: E731
    got = dict(logprobs=f(rows), stats=f(rows, 2), entropy=f(rows))
    size = max(tt.head_scores_workspace(rows, vocab, width), tt.head_scores_grad_workspace(rows, vocab, width))
    room = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    tt.head_scores(hidden, weight, t, workspace=room, **got)
    torch.cuda.synchronize()
    return z, off, exact(z), got, room


@pytest.mark.parametrize("kind", TYPES[1:])
@pytest.mark.parametrize("lift", [6.0, 15.0, 18.0, 21.0])
@pytest.mark.parametrize("rows,vocab,width", HEADS)
def test_head_scores_of_sure_rows(gpu, rows, vocab, width, kind, lift):
    hidden, weight, t = sure_head(rows, vocab, width, kind, lift)
    t[1::7] = -1
    z, off, e, got, _ = head_scores(hidden, weight, t)
    assert bool((z.argmax(1) == t)[t >= 0].all())
    tol = relative_error(e["depth"], vocab) + 2 * off
    near(got["stats"][:, 1], e["log_s"], tol * e["log_s"])
    # (the mean exponent carries the logits' errors as they stand)
    near(got["entropy"], e["entropy"], (2 * tol + 2 * off) * e["entropy"] + 2 * off * torch.expm1(e["log_s"]))
    given = torch.where(t < 0, torch.zeros_like(e["log_s"]), e["lp"].gather(1, t.clamp(min=0).long()[:, None])[:, 0])
    near(got["logprobs"], given, tol * given.abs())


@pytest.mark.parametrize("kind", TYPES[1:])
@pytest.mark.parametrize("lift", [6.0, 15.0, 18.0, 21.0])
@pytest.mark.parametrize("rows,vocab,width", HEADS)
def test_head_gradients_from_the_scores_own_statistics(gpu, rows, vocab, width, kind, lift):
    hidden, weight, t = sure_head(rows, vocab, width, kind, lift)
    t[1::7] = -1
    z, off, e, got, room = head_scores(hidden, weight, t)
    # gradients of the log probabilities, large enough that the results are ordinary 16-bit floats
    a = torch.full((rows,), 4096.0, device="cuda")
    gh, gw = torch.empty_like(hidden), torch.empty_like(weight)
    tt.head_scores_grad(hidden, weight, t, got["stats"], None, a, None, gh, gw, workspace=room)
    torch.cuda.synchronize()
    h, w = hidden.double(), weight.double()
    g, size = exact_grad(e, t, a.double(), torch.zeros_like(a).double())
    unit, least = ref.ROUNDING[kind]
    rel = 2 * relative_error(e["depth"], vocab) + 6 * off + 16 * ref.U32 + (unit if rows > 256 else 2.0**-16)
    floor = least * 2  # what is below the smallest 16-bit float beside a gradient of 4096
    want = g @ w
    near(gh, want, size @ w.abs() * (rel + vocab * ref.U32) + floor * w.abs().sum(0) + unit * want.abs() + least)
    want = g.t().contiguous() @ h
    near(gw, want, size.t().contiguous() @ h.abs() * (rel + rows * ref.U32) + floor * h.abs().sum(0) + unit * want.abs() + least)
