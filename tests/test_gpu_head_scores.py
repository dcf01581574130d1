"""Scores of hidden states through the head's weights, and the gradients, against 64 bits."""

import math

import pytest

torch = pytest.importorskip("torch")
import model_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


def make(rows, vocab, width, kind, seed, pad=0, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def matrix(n, spread):
        buf = torch.full((n, width + pad + shift), 77.0, dtype=kind, device="cuda")
        m = buf[:, shift:shift + width]
        m.copy_(torch.randn(n, width, generator=gen, device="cuda") * spread)
        return m

    hidden, weight = matrix(rows, 1.0), matrix(vocab, 2.5 / math.sqrt(width))
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    return hidden, weight, t


def exact_logits(hidden, weight):
    h, w = hidden.double(), weight.double()
    z = h @ w.t().contiguous()
    # a sum of `width` products in 32 bits, in any order
    return z, float((h.abs() @ w.t().contiguous().abs()).max()) * h.shape[1] * ref.U32


def run(hidden, weight, t, scale=1.0, stream=None):
    from paper_2607_29678_amd import head_scores, head_scores_workspace

    rows, vocab = len(hidden), len(weight)
    f = lambda *s: torch.full(s, 77.0, device="cuda")  # noqa: E731
    out = dict(logprobs=f(rows), stats=f(rows, 2), entropy=f(rows))
    work = torch.full((head_scores_workspace(rows, vocab, hidden.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    head_scores(hidden, weight, t, workspace=work, scale=scale, stream=stream, **out)
    torch.cuda.synchronize()
    return out


def check(hidden, weight, t, scale=1.0, **kw):
    got = run(hidden, weight, t, scale, **kw)
    z, off = exact_logits(hidden, weight)
    want = ref.scores(z, t, scale)
    deepest = ref.depth_of(want["lp"])
    tol = ref.score_error(len(weight), deepest, off * scale)
    ref.close(got["logprobs"], want["logprobs"], tol)
    ref.close(got["stats"][:, 0], want["stats"][:, 0], off)
    ref.close(got["stats"][:, 1], want["stats"][:, 1], tol)
    ref.close(got["entropy"], want["entropy"], 2 * tol * (1 + math.log(len(weight)) + deepest * 2.0 ** -10))
    return got


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 700])
def test_rows(gpu, kind, rows):
    check(*make(rows, 1281, 256, kind, rows))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 31, 127, 128, 129, 255, 257, 8449, 50257])
def test_vocabularies(gpu, kind, vocab):
    for rows in (3, 200):
        check(*make(rows, vocab, 128, kind, vocab))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("width", [1, 7, 8, 15, 16, 63, 64, 65, 72, 127, 200, 1000, 2048])
def test_widths(gpu, kind, width):
    for rows in (5, 40, 100, 300):
        check(*make(rows, 700, width, kind, width))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (8, 8), (5, 3)])
def test_strides(gpu, kind, pad, shift):
    for rows in (5, 300):
        check(*make(rows, 900, 128, kind, 7, pad, shift))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab,width", [(256, 50_257, 72), (250, 50_001, 520), (1000, 20_011, 64), (513, 60_003, 192)])
def test_many_tiles(gpu, kind, rows, vocab, width):
    """Enough tiles to fill the compute units, with both tile widths among them."""
    check(*make(rows, vocab, width, kind, rows))


def test_targets_and_scale(gpu):
    hidden, weight, t = make(300, 1281, 128, torch.bfloat16, 8)
    t[0], t[1], t[2], t[299] = -1, 1281, 1280, 0
    got = check(hidden, weight, t, 0.7)
    assert float(got["logprobs"][0]) == 0 and math.isnan(float(got["logprobs"][1]))
    none = run(hidden, weight, None, 0.7)
    assert bool((none["logprobs"] == 0).all()) and torch.equal(none["entropy"], got["entropy"])


def test_rows_without_a_distribution(gpu):
    for rows in (3, 300):
        hidden, weight, t = make(rows, 600, 64, torch.bfloat16, 9)
        hidden[1, 3] = math.nan
        got = run(hidden, weight, t)
        assert math.isnan(float(got["logprobs"][1])) and math.isnan(float(got["entropy"][1]))
        ok = [i for i in range(rows) if i != 1]
        assert bool(torch.isfinite(got["logprobs"][ok]).all())


def test_agrees_with_stored_logits(gpu):
    """Integers of a few bits multiply and add without rounding: both forms give the same logits."""
    from paper_2607_29678_amd import token_scores

    gen = torch.Generator(device="cuda").manual_seed(10)
    hidden = torch.randint(-3, 4, (150, 192), generator=gen, device="cuda").bfloat16()
    weight = torch.randint(-2, 3, (2000, 192), generator=gen, device="cuda").bfloat16()
    t = torch.randint(0, 2000, (150,), generator=gen, device="cuda", dtype=torch.int32)
    z = hidden.float() @ weight.float().t()
    got = run(hidden, weight, t, 0.05)
    lp, st = torch.zeros(150, device="cuda"), torch.zeros(150, 2, device="cuda")
    from paper_2607_29678_amd import token_scores_workspace
    work = torch.empty(max(1, token_scores_workspace(150, 2000, 0)), dtype=torch.uint8, device="cuda")
    token_scores(z, t, lp, st, scale=0.05, workspace=work, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(got["stats"][:, 0], st[:, 0])
    ref.close(got["logprobs"], lp.double(), 2 * ref.score_error(2000, 60))


def test_same_results_each_time(gpu):
    for rows in (4, 300):
        args = make(rows, 5000, 256, torch.bfloat16, 11)
        first = run(*args)
        for _ in range(3):
            again = run(*args)
            assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("rows", [5, 300])
def test_captured_head_on_new_inputs(gpu, rows):
    """Scores and gradients captured once follow what is in their inputs when they are replayed."""
    from paper_2607_29678_amd import head_scores, head_scores_grad, head_scores_grad_workspace, head_scores_workspace

    vocab, width = 3000, 128
    hidden, weight, t = make(rows, vocab, width, torch.bfloat16, 30)
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    lp, st, en = f(rows), f(rows, 2), f(rows)
    a, b = grads(rows)
    gh, gw = torch.zeros_like(hidden), torch.zeros_like(weight)
    size = max(head_scores_workspace(rows, vocab, width), head_scores_grad_workspace(rows, vocab, width))
    work = torch.empty(size, dtype=torch.uint8, device="cuda")

    def call():
        s = torch.cuda.current_stream().cuda_stream
        head_scores(hidden, weight, t, lp, st, en, workspace=work, stream=s)
        head_scores_grad(hidden, weight, t, st, en, a, b, gh, gw, workspace=work, stream=s)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        for dst, src in zip((hidden, weight, t), make(rows, vocab, width, torch.bfloat16, 40 + seed)):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (lp, st, en, gh, gw)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (lp, st, en, gh, gw)))
        check(hidden, weight, t)


def test_another_stream(gpu):
    s = torch.cuda.Stream()
    check(*make(70, 3000, 128, torch.bfloat16, 12), stream=s.cuda_stream)


# ---- gradients ----


def run_grad(hidden, weight, t, g_lp, g_e, scale=1.0, room=None, want_hidden=True, want_weight=True, outs=None):
    from paper_2607_29678_amd import head_scores_grad, head_scores_grad_workspace

    z, _ = exact_logits(hidden, weight)
    s = ref.scores(z, t, scale)
    rows, vocab, width = len(hidden), len(weight), hidden.shape[1]
    gh, gw = outs or (torch.full((rows, width), 55.0, dtype=hidden.dtype, device="cuda"),
                      torch.full((vocab, width), 55.0, dtype=hidden.dtype, device="cuda"))
    least, ample = (head_scores_grad_workspace(rows, vocab, width, x) for x in (False, True))
    assert least <= ample
    size = ample if room is None else least + int(room * (ample - least))
    work = torch.full((max(1, size),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    head_scores_grad(hidden, weight, t, s["stats"].float().contiguous(), None if g_e is None else s["entropy"].float(),
                     g_lp, g_e, gh if want_hidden else None, gw if want_weight else None, scale=scale, workspace=work,
                     stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return gh, gw


def grads(rows, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, generator=gen, device="cuda") / rows, torch.randn(rows, generator=gen, device="cuda") * 0.3 / rows)


def check_grad(hidden, weight, t, g_lp, g_e, scale=1.0, **kw):
    rows, vocab, width = len(hidden), len(weight), hidden.shape[1]
    z, off = exact_logits(hidden, weight)
    zero = torch.zeros(rows, dtype=torch.float64, device="cuda")
    a = zero if g_lp is None else g_lp.double()
    b = zero if g_e is None else g_e.double()
    g, size = ref.logits_grad(z, t, a, b, scale)
    h, w = hidden.double(), weight.double()
    gh, gw = run_grad(hidden, weight, t, g_lp, g_e, scale, **kw)
    unit, least = ref.ROUNDING[hidden.dtype]
    depth = float(ref.depth_of(ref.scores(z, t, scale)["lp"]).max())
    # an entry of G: the exponent (the logit's own error and the roundings), then its own rounding
    rel = 2 * off * scale * (1 + depth) + ref.U32 * (8 * depth + 8 * math.log(vocab) + 16) + unit
    floor = least * 2.0 ** -11 * float(size.max())  # what is below the smallest 16-bit float after G's scaling
    if kw.get("want_hidden", True):
        ah = size @ w.abs()
        want = g @ w
        ref.close(gh, want, ah * (rel + vocab * ref.U32) + floor * w.abs().sum(0) + unit * want.abs() + least)
    if kw.get("want_weight", True):
        aw = size.t().contiguous() @ h.abs()
        want = g.t().contiguous() @ h
        ref.close(gw, want, aw * (rel + rows * ref.U32) + floor * h.abs().sum(0) + unit * want.abs() + least)
    return gh, gw


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 255, 257, 600])
def test_grad_rows(gpu, kind, rows):
    check_grad(*make(rows, 1281, 256, kind, rows), *grads(rows))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 63, 255, 256, 257, 8449])
def test_grad_vocabularies(gpu, kind, vocab):
    check_grad(*make(100, vocab, 128, kind, vocab), *grads(100))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("width", [1, 7, 8, 64, 65, 200, 513])
def test_grad_widths(gpu, kind, width):
    check_grad(*make(90, 700, width, kind, width), *grads(90))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab,width", [(256, 50_257, 72), (250, 50_001, 1024), (1000, 20_011, 64), (513, 60_003, 192)])
def test_grad_many_tiles(gpu, kind, rows, vocab, width):
    """Enough tiles to fill the compute units, with both tile widths among them."""
    check_grad(*make(rows, vocab, width, kind, rows), *grads(rows))


@pytest.mark.parametrize("room", [0.0, 0.2, 0.5, 0.99])
def test_grad_in_pieces(gpu, room):
    """Less workspace: the vocabulary in several pieces, the last one shorter."""
    check_grad(*make(130, 3001, 192, torch.bfloat16, 20), *grads(130), room=room)


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_grad_strides(gpu, pad, shift):
    hidden, weight, t = make(70, 900, 128, torch.bfloat16, 21, pad, shift)
    bh = torch.full((70, 128 + 9), 55.0, dtype=torch.bfloat16, device="cuda")
    bw = torch.full((900, 128 + 9), 55.0, dtype=torch.bfloat16, device="cuda")
    check_grad(hidden, weight, t, *grads(70), outs=(bh[:, 5:133], bw[:, 2:130]))
    for b, lo, hi in ((bh, 5, 133), (bw, 2, 130)):
        assert bool((b[:, :lo] == 55).all()) and bool((b[:, hi:] == 55).all())


@pytest.mark.parametrize("kind", TYPES)
def test_grad_of_one_side(gpu, kind):
    args = make(100, 1281, 128, kind, 22)
    a, b = grads(100)
    gh, gw = check_grad(*args, a, b, want_weight=False)
    assert bool((gw == 55).all())
    gh, gw = check_grad(*args, a, b, want_hidden=False)
    assert bool((gh == 55).all())
    check_grad(*args, a, None)
    check_grad(*args, None, b)


def test_grad_of_given_tokens_only(gpu):
    hidden, weight, t = make(200, 1000, 64, torch.bfloat16, 23)
    t[::3] = -1
    a, _ = grads(200)
    gh, _ = check_grad(hidden, weight, t, a, None)
    assert bool((gh[::3] == 0).all())


@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e4])
def test_grad_of_any_size_in_f16(gpu, size):
    """G is scaled into the 16-bit range: only the results' own range limits them (1e4: to about 1e4)."""
    hidden, weight, t = make(64, 600, 64, torch.float16, 24)
    a, b = grads(64)
    check_grad(hidden, weight, t, a * size, b * size)


def test_grad_of_no_rows(gpu):
    hidden = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    _, weight, _ = make(1, 300, 64, torch.bfloat16, 25)
    e = torch.empty(0, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    gw = torch.full((300, 64), 55.0, dtype=torch.bfloat16, device="cuda")
    from paper_2607_29678_amd import head_scores_grad
    head_scores_grad(hidden, weight, t, torch.empty(0, 2, device="cuda"), e, e, e, torch.empty_like(hidden), gw,
                     stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert bool((gw == 0).all())


def test_grad_against_differences(gpu):
    """<gradient, v> against central differences of the forward kernel; all points are 16-bit floats exactly."""
    rows, vocab, width, step = 30, 200, 32, 2.0 ** -5
    gen = torch.Generator(device="cuda").manual_seed(26)
    grid = lambda n: torch.randint(-16, 17, (n, width), generator=gen, device="cuda") / 16.0  # noqa: E731
    sign = lambda n: torch.randint(-1, 2, (n, width), generator=gen, device="cuda").float()  # noqa: E731
    hidden, weight, vh, vw = grid(rows), grid(vocab), sign(rows), sign(vocab)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    t[::9] = -1
    a, b = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda") * 0.3

    def value(h, w):
        for m in (h, w):
            assert torch.equal(m.half().float(), m)
        o = run(h.half(), w.half(), t)
        return float((a.double() * o["logprobs"].double() + b.double() * o["entropy"].double()).sum())

    gh, gw = run_grad(hidden.half(), weight.half(), t, a, b)
    _, size = ref.logits_grad(hidden.double() @ weight.double().t().contiguous(), t, a.double(), b.double())
    terms = (size @ weight.double().abs(), size.t().contiguous() @ hidden.double().abs())
    for which, v, g in ((0, vh, gh), (1, vw, gw)):
        at = lambda e: value(hidden + e * v, weight) if which == 0 else value(hidden, weight + e * v)  # noqa: E731,B023
        numeric = (at(step) - at(-step)) / (2 * step)
        half = (at(2 * step) - at(-2 * step)) / (4 * step)
        formula = float((g.double() * v.double()).sum())
        # the step's own error is a third of what doubling the step changes, with as much again for the next order;
        # the entries of G and the results are rounded to 11 bits, values carry 1e-5 each
        rounding = 2.0 ** -11 * float(((terms[which] + g.double().abs()) * v.abs()).sum())
        tol = 2 * abs(half - numeric) / 3 + rounding + rows * 2e-5 / step
        assert abs(numeric - formula) <= tol, (which, numeric, formula, tol)


def test_grad_offsets_past_32_bits(gpu):
    """Weights of more than 2^31 entries: the last rows take part."""
    width, vocab, rows = 8192, 270_000, 8
    weight = torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(27)
    weight[-5:] = (torch.randn(5, width, generator=gen, device="cuda") * 0.02).bfloat16()
    hidden = torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    t = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    t[0] = vocab - 3
    got = run(hidden, weight, t)
    tail = hidden.double() @ weight[-5:].double().t().contiguous()
    lse = torch.logsumexp(torch.cat([tail, torch.full((rows, 1), math.log(vocab - 5), dtype=torch.float64, device="cuda")], 1), 1)
    given = tail.gather(1, (t.long() - (vocab - 5))[:, None])[:, 0]
    _, off = exact_logits(hidden, weight[-5:])
    ref.close(got["logprobs"], given - lse, ref.score_error(vocab, 20, off))
    from paper_2607_29678_amd import head_scores_grad, head_scores_grad_workspace
    gh = torch.zeros_like(hidden)
    work = torch.empty(head_scores_grad_workspace(rows, vocab, width, False) + (256 << 20), dtype=torch.uint8, device="cuda")
    a = torch.ones(rows, device="cuda")
    gw = torch.empty_like(weight)
    head_scores_grad(hidden, weight, t, got["stats"], None, a, None, gh, gw, workspace=work,
                     stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    p = (tail - lse[:, None]).exp()
    g = -p
    g[torch.arange(rows, device="cuda"), t.long() - (vocab - 5)] += 1
    want = g @ weight[-5:].double()
    unit = 2.0 ** -8
    size = g.abs() + p
    ref.close(gh, want, (size @ weight[-5:].double().abs()) * (2 * unit + 2 * off + 1e-4) + unit * want.abs() + 1e-9)
    want = g.t().contiguous() @ hidden.double()
    ref.close(gw[-5:], want, (size.t().contiguous() @ hidden.double().abs()) * (2 * unit + 2 * off + 1e-4) + unit * want.abs() + 1e-9)
