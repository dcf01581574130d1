"""Gradients where rounding shows most: a given token that is nearly sure, and a few rows whose errors do not average out."""

import math

import pytest

torch = pytest.importorskip("torch")
import paper_2607_29678_amd as tt  # noqa: E402

pytestmark = pytest.mark.gpu


def exact_gradient(z, targets, a, b):
    """Of sum(a logprob + b entropy) with respect to z, in 64 bits."""
    lp = z.log_softmax(1)
    p = lp.exp()
    plogp = p * lp
    rows = torch.arange(len(z), device=z.device)
    a = torch.where(targets < 0, torch.zeros_like(a), a)
    g = -p * a[:, None]
    # (1 - p of the given token, without the cancellation)
    t = targets.clamp(min=0).long()
    g[rows, t] = torch.where(targets < 0, g[rows, t], -a * torch.expm1(lp[rows, t]))
    return g - b[:, None] * (plogp - p * plogp.sum(1, keepdim=True))


def statistics(z):
    """{m, log s} and the entropy, rounded once from 64 bits."""
    m = z.amax(1)
    t = z.argmax(1, keepdim=True)
    e = (z - m[:, None]).exp()
    log_s = torch.log1p(e.scatter(1, t, 0.0).sum(1))
    lp = z.log_softmax(1)
    return torch.stack([m, log_s], 1).float(), (-(lp.exp() * lp).sum(1)).float()


@pytest.mark.parametrize("entropy_weight", [0.0, 0.25])
@pytest.mark.parametrize("lift", [4.0, 18.0, 22.0])
@pytest.mark.parametrize("rows,vocab,given", [(1, 1_281, 0), (1, 1_281, 1_280), (3, 1_000, 517), (2, 8_449, 4_000)])
def test_sure_token(rows, vocab, given, lift, entropy_weight):
    # At the given token d = -log2 s is off by two roundings, exp and expm1 by two units: 8 roundings with the
    # products, 5e-7 of its value, and the entropy's part by as much of its own terms p (log p + entropy) after
    # log p + entropy was rounded: 2^-23 (|log p| + entropy) of p.  Elsewhere d (below 60) carries three roundings:
    # 60 * 3 * 2^-24 of p.
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = (torch.randn(rows, vocab, generator=gen, device="cuda") * 2.0).clamp(max=8.0)
    x[:, given] = lift
    z = x.double()
    targets = torch.full((rows,), given, dtype=torch.int32, device="cuda")
    a = torch.linspace(0.7, 1.3, rows, device="cuda")
    b = torch.full((rows,), entropy_weight, device="cuda")
    stats, entropy = statistics(z)
    out = torch.empty_like(x)
    tt.token_scores_grad(x, targets, stats, entropy, a, b, out)
    torch.cuda.synchronize()
    want = exact_gradient(z, targets, a.double(), b.double())
    lp = z.log_softmax(1)
    p, h = lp.exp(), entropy.double()[:, None]
    room = 5e-7 * want.abs() + entropy_weight * p * (2.0**-20 * (lp.abs() + h))
    other = torch.arange(vocab, device="cuda") != given
    room += other * (a[:, None] + entropy_weight * (lp.abs() + h)) * p * 1.1e-5
    off = (out.double() - want).abs()
    assert bool((off <= room).all()), float((off / room).max())


@pytest.mark.parametrize("ample", [True, False])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,vocab,width", [(1, 1_003, 256), (2, 2_049, 250), (8, 4_001, 256), (63, 2_000, 512), (64, 1_500, 128),
                                              (65, 1_500, 136), (129, 900, 77), (256, 1_025, 256)])
def test_few_rows_keep_their_products(rows, vocab, width, kind, ample):
    # G in two parts is good to 2^-17 or better, the recomputed logits (below 20, 32-bit sums) to some 2e-5 of p: next to
    # the results' own rounding (2^-9 and 2^-12 in the mean, at least) these add less than a tenth.
    gen = torch.Generator(device="cuda").manual_seed(rows)
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    weight = (torch.randn(vocab, width, generator=gen, device="cuda") * (2.0 / math.sqrt(width))).to(kind)
    hidden = (torch.randn(rows, width, generator=gen, device="cuda") + weight[targets.long()].float()).to(kind)
    if rows > 2:
        targets[rows // 2] = -1
    a = torch.randn(rows, generator=gen, device="cuda") + 0.1
    b = torch.full((rows,), 0.01, device="cuda")
    h, w = hidden.double(), weight.double()
    z = h @ w.t().contiguous()
    stats, entropy = statistics(z)
    room = torch.empty(tt.head_scores_grad_workspace(rows, vocab, width, ample), dtype=torch.uint8, device="cuda")
    room.fill_(255)  # (not a number, wherever the call should read none of it)
    gh, gw = torch.empty_like(hidden), torch.empty_like(weight)
    tt.head_scores_grad(hidden, weight, targets, stats, entropy, a, b, gh, gw, workspace=room)
    torch.cuda.synchronize()
    g = exact_gradient(z, targets, a.double(), b.double())
    for got, want in ((gh, g @ w), (gw, g.t().contiguous() @ h)):
        rounding = (want.to(kind).double() - want).norm()
        off = (got.double() - want).norm()
        assert float(off) <= 1.1 * float(rounding), float(off / rounding)
