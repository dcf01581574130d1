"""Head gradients as a whole: the norm of their error next to that of the results' own rounding.

A bound of every entry has to allow for all terms being off at once; the norm of the error does not, and shows a stage
of a sum that is left out, a part that is not added or a term of the formula that is missing.
"""

import math

import pytest

torch = pytest.importorskip("torch")
import paper_2607_29678_amd as tt  # noqa: E402

TYPES = [torch.bfloat16, torch.float16]
# Up to 256 rows G is good to 2^-16 and adds less than a tenth to the results' own rounding.  More rows: every entry of G
# is rounded as the results are, and as the errors are independent the norm grows by sqrt 2, with a fifth on top for the
# few rows whose one large entry decides.
FEW, MANY = 1.1, 1.7


def make(rows, vocab, width, kind, device, seed=6):
    gen = torch.Generator(device=device).manual_seed(seed + rows)
    # given tokens are dealt over the vocabulary, one in `rows` of it each
    t = (torch.arange(rows, device=device) * vocab // rows).to(torch.int32)
    t = t[torch.randperm(rows, generator=gen, device=device)]
    weight = (torch.randn(vocab, width, generator=gen, device=device) * (2.0 / math.sqrt(width))).to(kind)
    hidden = (torch.randn(rows, width, generator=gen, device=device) + weight[t.long()].float()).to(kind)
    a = torch.randn(rows, generator=gen, device=device) / rows
    b = (torch.rand(rows, generator=gen, device=device) + 0.5) / rows
    return hidden, weight, t, a, b


def softmax(hidden, weight):
    z = hidden.double() @ weight.double().t().contiguous()
    return z, z.log_softmax(1)


def gradient(lp, t, a, b):
    """Of sum(a logprob + b entropy) with respect to the logits; either may be None."""
    p = lp.exp()
    g = torch.zeros_like(p)
    if a is not None:
        g -= p * a.double()[:, None]
        g[torch.arange(len(p), device=p.device), t.long()] += a.double()
    if b is not None:
        g -= b.double()[:, None] * p * (lp - (p * lp).sum(1, keepdim=True))
    return g


def off_by(got, want, kind):
    """The error's norm in units of the norm of what rounding the exact result takes off."""
    want = want.double()
    return float((got.double() - want).norm() / (want.to(kind).double() - want).norm())


# ---- that the measure sees what it should, with mistakes planted in a plain form (no GPU) ----


@pytest.mark.parametrize("mistake,shown", [(None, False), ("stage", True), ("rows", True), ("entropy", True), ("given", True)])
def test_the_norm_shows_mistakes(mistake, shown):
    rows, vocab, width, kind = 300, 12_003, 64, torch.bfloat16
    hidden, weight, t, a, b = make(rows, vocab, width, kind, "cpu")
    _, lp = softmax(hidden, weight)
    worst = 0.0
    for aa, bb in ((a, None), (None, b), (a, b)):
        g = gradient(lp, t, aa, bb)
        bad = gradient(lp, t, aa, None if mistake == "entropy" and bb is not None else bb)
        if mistake == "given" and aa is not None:
            bad[torch.arange(rows), t.long()] -= aa.double()
        bad = bad.to(kind).double()
        n, k = slice(0, vocab), slice(0, rows)
        if mistake == "stage":  # 64 entries of the sum over the vocabulary
            bad = bad.clone()
            cut = bad.clone()
            cut[:, 6_400:6_464] = 0
            gh = cut @ weight.double()
        else:
            gh = bad[:, n] @ weight.double()
        if mistake == "rows":  # a stage of the sum over the rows
            k = slice(64, rows)
        gw = bad[k].t() @ hidden.double()[k]
        worst = max(worst, off_by(gh.to(kind), g @ weight.double(), kind), off_by(gw.to(kind), g.t() @ hidden.double(), kind))
    assert (worst > MANY) == shown, worst


# ---- the kernels ----


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("room", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("rows,vocab,width", [(250, 50_001, 1024), (256, 50_257, 72), (257, 50_001, 256), (513, 60_003, 192),
                                              (640, 20_011, 1000), (1000, 20_011, 64), (300, 9_001, 333), (2_048, 8_449, 512)])
def test_norm_of_the_error(gpu, rows, vocab, width, kind, room):
    hidden, weight, t, a, b = make(rows, vocab, width, kind, "cuda")
    z, lp = softmax(hidden, weight)
    m = z.amax(1)
    stats = torch.stack([m, (z - m[:, None]).exp().sum(1).log()], 1).float()
    entropy = -(lp.exp() * lp).sum(1).float()
    least, ample = (tt.head_scores_grad_workspace(rows, vocab, width, x) for x in (False, True))
    work = torch.full((least + int(room * (ample - least)),), 255, dtype=torch.uint8, device="cuda")
    h, w = hidden.double(), weight.double()
    for aa, bb in ((a, None), (None, b), (a, b)):
        g = gradient(lp, t, aa, bb)
        gh, gw = torch.full_like(hidden, 55.0), torch.full_like(weight, 55.0)
        tt.head_scores_grad(hidden, weight, t, stats, entropy, aa, bb, gh, gw, workspace=work)
        torch.cuda.synchronize()
        most = FEW if rows <= 256 else MANY
        off = off_by(gh, g @ w, kind), off_by(gw, g.t().contiguous() @ h, kind)
        assert max(off) <= most, off
