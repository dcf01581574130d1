"""Scores of stored logits and their gradient against 64 bits."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import model_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF = math.inf


def logits_of(rows, vocab, kind, seed, pad=0, shift=0, spread=2.5):
    """Rows of logits inside a wider buffer, ``shift`` entries from its start."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows, vocab + pad + shift), 99.0, dtype=kind, device="cuda")
    z = buf[:, shift:shift + vocab]
    z.copy_(torch.randn(rows, vocab, generator=gen, device="cuda") * spread)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    return z, t


def run(z, t, n_alt=0, scale=1.0, stream=None):
    from paper_2607_29678_amd import token_scores, token_scores_workspace

    rows, vocab = z.shape
    f = lambda *s: torch.full(s, 77.0, device="cuda")  # noqa: E731
    out = dict(logprobs=f(rows), stats=f(rows, 2), entropy=f(rows))
    if n_alt:
        out.update(alt_ids=torch.full((rows, n_alt), -77, dtype=torch.int32, device="cuda"), alt_logprobs=f(rows, n_alt))
    need = token_scores_workspace(rows, vocab, n_alt)
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    torch.cuda.synchronize()
    token_scores(z, t, scale=scale, workspace=work, stream=stream, **out)
    torch.cuda.synchronize()
    return out


def check(z, t, n_alt=0, scale=1.0, **kw):
    got = run(z, t, n_alt, scale, **kw)
    want = ref.scores(z.double(), t, scale, n_alt)
    deepest = ref.depth_of(want["lp"])
    tol = ref.score_error(z.shape[1], deepest)
    own = 4 * ref.U32  # a log probability's own roundings
    ref.close(got["logprobs"], want["logprobs"], tol + own * want["logprobs"].abs())
    # the largest logit is one of the row's; the logarithm of the sum has no exponent of its own
    assert torch.equal(torch.nan_to_num(got["stats"][:, 0].double(), nan=1e300), torch.nan_to_num(want["stats"][:, 0], nan=1e300))
    ref.close(got["stats"][:, 1], want["stats"][:, 1], tol)
    # entropy: the weights' relative error once on log s, once on the mean exponent
    ref.close(got["entropy"], want["entropy"], 2 * tol * (1 + math.log(z.shape[1]) + deepest * 2.0 ** -10))
    if n_alt:
        assert torch.equal(got["alt_ids"].cpu().long(), want["alt_ids"])
        ref.close(got["alt_logprobs"], want["alt_logprobs"], tol.cpu()[:, None] + own * want["alt_logprobs"].abs())
    return got


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 257, 1281, 2047, 4099, 8449, 50257])
def test_vocabularies(gpu, kind, vocab):
    z, t = logits_of(5, vocab, kind, vocab)
    for n_alt in (0, 1, 5, 64):
        check(z, t, n_alt)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 3, 100, 1023, 1024, 1500])
def test_rows(gpu, kind, rows):
    z, t = logits_of(rows, 8449, kind, rows)
    check(z, t, 20)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shift,pad", [(1, 0), (3, 2), (5, 64), (0, 7)])
def test_rows_at_any_alignment(gpu, kind, shift, pad):
    for rows, vocab in ((33, 5003), (1100, 517)):
        z, t = logits_of(rows, vocab, kind, shift + pad, pad, shift)
        check(z, t, 8)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [4, 1030])
def test_masked_rows(gpu, kind, rows):
    """-inf and the type's lowest value as masks; few, one or no entries left."""
    vocab = 8449
    z, t = logits_of(rows, vocab, kind, 11)
    low = torch.finfo(kind).min
    whole = z.clone()
    for i, (mask, left) in enumerate([(-INF, 3), (low, 3), (-INF, 0), (low, 0), (-INF, 1), (low, 40), (-INF, 4000)]):
        r = i % rows if rows < 7 else i * (rows // 7)
        z[r] = mask
        keep = torch.randperm(vocab, generator=torch.Generator().manual_seed(i))[:left].to("cuda")
        z[r, keep] = whole[r, keep]
        if rows < 7:
            check(z, t, 20)
    check(z, t, 20)


@pytest.mark.parametrize("kind", TYPES)
def test_ties(gpu, kind):
    """Equal entries are taken in order of their IDs, also where nearly all of a row is equal."""
    vocab = 20_011
    z, t = logits_of(6, vocab, kind, 12)
    z[0] = 1.5
    z[1] = 0.0
    z[1, 1::2] = -0.0
    z[2, 5000:] = 3.0
    z[3] = torch.round(z[3].float()).to(kind)
    z[4] = -2.0
    z[4, -3:] = 4.0
    check(z, t, 64)
    check(z, t, 1)
    big = z.repeat(200, 1)
    check(big, t.repeat(200), 9)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [2, 1025])
def test_sorted_rows(gpu, kind, rows):
    """Rows in rising order put every later entry among the candidates; in a strided order, all in one thread."""
    vocab = 50_257
    z = torch.sort(torch.randn(rows, vocab, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda"), 1).values
    t = torch.arange(rows, dtype=torch.int32, device="cuda")
    check(z.to(kind), t, 20)
    check(z.flip(1).to(kind).contiguous(), t, 20)


def test_one_thread_holds_all_large_entries(gpu):
    vocab = 8 * 256 * 4 * 40
    z = torch.zeros(1030, vocab, dtype=torch.bfloat16, device="cuda")
    cols = torch.arange(vocab, device="cuda")
    mine = (cols // 8) % 256 == 17  # one thread's vectors where a block takes a whole row
    z[:, mine] = (torch.arange(int(mine.sum()), device="cuda") % 120).bfloat16() + 1
    check(z[:, :].contiguous()[:1025], torch.zeros(1025, dtype=torch.int32, device="cuda"), 64)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [5, 1030])
def test_rows_without_a_distribution(gpu, kind, rows):
    z, t = logits_of(rows, 4100, kind, 13)
    z[0] = -INF
    z[1, 77] = math.nan
    z[2, 4099] = INF
    z[3] = math.nan
    t[0] = 5
    check(z, t, 4)
    t[0] = -1
    got = check(z, t, 4)
    assert float(got["logprobs"][0]) == 0.0 and float(got["entropy"][0]) == 0.0


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab,shift", [(4099, 0), (1281, 3), (65, 1), (9001, 0)])
def test_many_short_rows(gpu, kind, vocab, shift):
    """Rows that one wave takes, with masks, ties, sorted rows and rows without a distribution among them."""
    rows = 2100
    z, t = logits_of(rows, vocab, kind, vocab, 2, shift)
    whole = z.clone()
    low = torch.finfo(kind).min
    z[0] = -INF
    z[1] = low
    z[2] = 1.5
    z[3] = torch.sort(z[3].float()).values.to(kind)
    z[4] = torch.sort(z[4].float(), descending=True).values.to(kind)
    z[5, vocab // 2] = math.nan
    z[6, vocab - 1] = INF
    for r, (mask, left) in enumerate([(-INF, 3), (low, 3), (-INF, 1), (low, vocab // 2), (-INF, vocab // 2)], 7):
        z[r] = mask
        keep = torch.randperm(vocab, generator=torch.Generator().manual_seed(r))[:left].to("cuda")
        z[r, keep] = whole[r, keep]
    z[20:40] = torch.round(z[20:40].float()).to(kind)
    z[41] = 0.0
    z[41, 1::2] = -0.0
    cols = torch.arange(vocab, device="cuda")
    z[42] = torch.where((cols // (16 // z.element_size())) % 64 == 5, cols.float() % 50 + 1, torch.zeros(vocab, device="cuda")).to(kind)
    for n_alt in (0, 1, 20, 64):
        check(z, t, n_alt)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab,shift", [(24, 41_003, 0), (24, 24_576, 3), (60, 60_001, 1), (200, 82_001, 0), (450, 111_001, 5)])
def test_long_rows_in_parts(gpu, kind, rows, vocab, shift):
    """Rows that several blocks share: masks of whole parts, ties across them, sorted rows, rows without a distribution."""
    z, t = logits_of(rows, vocab, kind, vocab, 1, shift)
    whole = z.clone()
    low = torch.finfo(kind).min
    z[0] = -INF
    z[1] = low
    z[2] = 1.5
    z[3] = torch.sort(z[3].float()).values.to(kind)
    z[4] = torch.sort(z[4].float(), descending=True).values.to(kind)
    z[5, vocab // 2] = math.nan
    z[6, vocab - 1] = INF
    z[7, : vocab // 2] = -INF
    z[8, vocab // 7:] = low
    z[9, :-1] = -INF
    z[10, 1:] = -INF
    z[11] = 0.0
    z[11, 1::2] = -0.0
    z[12] = torch.round(z[12].float()).to(kind)
    for r, (mask, left) in enumerate([(-INF, 3), (low, 3), (-INF, 1), (low, vocab // 2), (-INF, vocab // 2), (low, 70)], 13):
        z[r] = mask
        keep = torch.randperm(vocab, generator=torch.Generator().manual_seed(r))[:left].to("cuda")
        z[r, keep] = whole[r, keep]
    z[20, ::700] = 9.0
    z[21, -64:] = 9.0
    z[22, :100] = torch.linspace(5, 8, 100, device="cuda").to(kind)
    for n_alt in (0, 1, 20, 64):
        check(z, t, n_alt)


def test_targets(gpu):
    z, t = logits_of(40, 1281, torch.float32, 14)
    t[3], t[4], t[5], t[6] = -1, -2**31, 1281, 2**31 - 1
    z[7, 9] = -INF
    t[7] = 9
    got = check(z, t)
    assert float(got["logprobs"][3]) == 0 and math.isnan(float(got["logprobs"][5])) and float(got["logprobs"][7]) == -INF
    none = run(z, None)
    assert bool((none["logprobs"] == 0).all()) and torch.equal(none["entropy"], got["entropy"])


def test_extreme_logits(gpu):
    z = torch.zeros(6, 3000, device="cuda")
    z[0] = 3e38
    z[1] = torch.linspace(-3e38, 3e38, 3000)
    z[2] = -3e38
    z[2, 5] = 3e38
    z[3] = torch.linspace(0, 1e-38, 3000)
    z[4] = 1e4 + torch.arange(3000) / 1024
    z[5, 0] = 80.0
    t = torch.tensor([1, 2999, 5, 0, 2999, 0], dtype=torch.int32, device="cuda")
    got = run(z, t, 3)
    want = ref.scores(z.double(), t, 1.0, 3)
    ref.close(got["logprobs"], want["logprobs"], ref.score_error(3000, 80) + 4 * ref.U32 * want["logprobs"].abs())
    ref.close(got["entropy"], want["entropy"], 20 * ref.score_error(3000, 80))
    assert torch.equal(got["alt_ids"].cpu().long(), want["alt_ids"])


@pytest.mark.parametrize("scale", [0.25, 1.7, 10.0])
def test_scale(gpu, scale):
    for kind in TYPES:
        z, t = logits_of(20, 8449, kind, 15)
        check(z, t, 7, scale)


def test_outputs_are_optional(gpu):
    from paper_2607_29678_amd import token_scores

    z, t = logits_of(1100, 600, torch.bfloat16, 16)
    want = run(z, t)
    for name in ("logprobs", "stats", "entropy"):
        got = torch.zeros_like(want[name])
        token_scores(z, t, **{name: got}, stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want[name])


def test_same_results_each_time(gpu):
    for rows in (3, 1100):
        z, t = logits_of(rows, 50257, torch.bfloat16, 17)
        first = run(z, t, 20)
        for _ in range(3):
            again = run(z, t, 20)
            assert all(torch.equal(first[k], again[k]) for k in first)


def test_offsets_past_32_bits(gpu):
    """The last rows of a matrix of more than 2^31 entries."""
    rows, vocab = 26_000, 100_257
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    part, t3 = logits_of(3, vocab, torch.bfloat16, 18)
    z[-3:] = part
    t = torch.zeros(rows, dtype=torch.int32, device="cuda")
    t[-3:] = t3
    got = run(z, t, 5)
    want = ref.scores(part.double(), t3, 1.0, 5)
    ref.close(got["logprobs"][-3:], want["logprobs"], ref.score_error(vocab, 40))
    assert torch.equal(got["alt_ids"][-3:].cpu().long(), want["alt_ids"])


# ---- gradient ----


def run_grad(z, t, g_lp, g_e, scale=1.0, out=None, stream=None):
    from paper_2607_29678_amd import token_scores_grad

    want = ref.scores(z.double(), t, scale)
    stats, entropy = want["stats"].float().contiguous(), want["entropy"].float()
    out = torch.full_like(z, 55.0, memory_format=torch.contiguous_format) if out is None else out
    torch.cuda.synchronize()
    token_scores_grad(z, t, stats, entropy if g_e is not None else None, g_lp, g_e, out, scale=scale, stream=stream)
    torch.cuda.synchronize()
    return out


def grads(rows, seed=1, entropy=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.randn(rows, generator=gen, device="cuda")
    b = torch.randn(rows, generator=gen, device="cuda") * 0.3
    return a, b if entropy else None


def check_grad(z, t, g_lp, g_e, scale=1.0, **kw):
    rows = len(z)
    x = z.double().clone()  # (the output may be z)
    zero = torch.zeros(rows, dtype=torch.float64, device="cuda")
    want, size = ref.logits_grad(x, t, zero if g_lp is None else g_lp.double(), zero if g_e is None else g_e.double(), scale)
    got = run_grad(z, t, g_lp, g_e, scale, **kw)
    lp = ref.scores(x, t, scale)["lp"]
    depth = torch.where(torch.isfinite(lp), -lp, torch.zeros_like(lp)).clamp(max=200)
    # the exponent has five roundings of values up to its depth and the two statistics, then 2 units of the exponential
    rel = ref.U32 * (8 * depth + 8 * math.log(z.shape[1]) + 16)
    unit, least = ref.ROUNDING[z.dtype]
    ref.close(got, want, size * rel + unit * want.abs() + least + 1e-37)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 65, 1281, 8192, 8449, 16384, 16385, 50257])
def test_grad_vocabularies(gpu, kind, vocab):
    z, t = logits_of(9, vocab, kind, vocab)
    t[1] = -1
    check_grad(z, t, *grads(9))
    check_grad(z, t, *grads(9, entropy=False))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 100_257), (70, 100_257), (700, 33_000), (4097, 1281), (4100, 20_011)])
def test_grad_rows(gpu, kind, rows, vocab):
    """One block a row, several blocks a row, several steps a block."""
    z, t = logits_of(rows, vocab, kind, rows)
    check_grad(z, t, *grads(rows))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shift,pad,out_shift,out_pad", [(1, 0, 0, 0), (3, 2, 3, 2), (0, 5, 2, 0), (2, 64, 1, 9)])
def test_grad_at_any_alignment(gpu, kind, shift, pad, out_shift, out_pad):
    rows, vocab = 37, 9001
    z, t = logits_of(rows, vocab, kind, 21, pad, shift)
    buf = torch.full((rows, vocab + out_pad + out_shift), 55.0, dtype=kind, device="cuda")
    check_grad(z, t, *grads(rows), out=buf[:, out_shift:out_shift + vocab])
    assert bool((buf[:, :out_shift] == 55).all()) and bool((buf[:, out_shift + vocab:] == 55).all())


@pytest.mark.parametrize("kind", TYPES)
def test_grad_in_place(gpu, kind):
    z, t = logits_of(50, 8449, kind, 22, 3, 1)
    check_grad(z, t, *grads(50), out=z)


@pytest.mark.parametrize("kind", TYPES)
def test_grad_of_masked_rows(gpu, kind):
    z, t = logits_of(8, 5000, kind, 23)
    keep = z.clone()
    z[0] = -INF
    z[1] = -INF
    z[1, 4:9] = keep[1, 4:9]
    t[1] = 5
    z[2] = torch.finfo(kind).min
    z[2, 100:103] = keep[2, 100:103]
    t[2] = 100
    z[3] = torch.finfo(kind).min
    z[4, 7] = -INF
    t[4] = 7
    check_grad(z, t, *grads(8))


def test_grad_of_rows_that_are_not_wanted(gpu):
    """No token given and no entropy gradient: exact zeros, whatever the row holds."""
    z, t = logits_of(4, 3000, torch.bfloat16, 24)
    t[:2] = -1
    z[1, 5] = math.nan
    got = run_grad(z, t, grads(4)[0], None)
    assert bool((got[:2] == 0).all()) and bool((got[2:] != 0).any())
    none = run_grad(z, t, None, None)
    assert bool((none == 0).all())


def test_grad_of_rows_without_a_distribution(gpu):
    z, t = logits_of(4, 3000, torch.float32, 25)
    z[0, 5] = math.nan
    z[1, 5] = INF
    t[2] = 3000
    got = run_grad(z, t, *grads(4))
    assert bool(torch.isnan(got[:3]).all()) and bool(torch.isfinite(got[3]).all())


def test_grad_scale(gpu):
    z, t = logits_of(12, 1281, torch.float32, 26)
    check_grad(z, t, *grads(12), scale=0.6)


def test_grad_against_differences(gpu):
    """<gradient, v> against central differences of the forward kernel along v."""
    rows, vocab, step = 40, 300, 2.0 ** -6
    z, t = logits_of(rows, vocab, torch.float32, 27)
    t[::7] = -1
    a, b = grads(rows, 3)
    v = torch.randn(rows, vocab, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")

    def value(x):
        o = run(x, t)
        return a.double() * o["logprobs"].double() + b.double() * o["entropy"].double()

    numeric = (value(z + step * v) - value(z - step * v)) / (2 * step)
    g = run_grad(z, t, a, b)
    formula = (g.double() * v.double()).sum(1)
    # third derivatives of log sum exp and of the entropy along v stay below about 6 |v|_inf^3 (1 + log vocab);
    # the values carry an error of about 1e-5, twice, over 2 steps
    tol = step**2 / 6 * 6 * float(v.abs().max())**3 * (1 + math.log(vocab)) + 1e-5 / step
    ref.close(numeric, formula, tol * (a.abs() + b.abs()).double() + 1e-9)


def test_captured_scores_on_new_logits(gpu):
    from paper_2607_29678_amd import token_scores, token_scores_grad, token_scores_workspace

    rows, vocab = 6, 50_257
    z, t = logits_of(rows, vocab, torch.bfloat16, 28)
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    lp, st, en, al = f(rows), f(rows, 2), f(rows), f(rows, 5)
    ai = torch.zeros(rows, 5, dtype=torch.int32, device="cuda")
    a, b = grads(rows)
    g = torch.zeros_like(z)
    work = torch.empty(token_scores_workspace(rows, vocab, 5), dtype=torch.uint8, device="cuda")

    def call():
        s = torch.cuda.current_stream().cuda_stream
        token_scores(z, t, lp, st, en, ai, al, workspace=work, stream=s)
        token_scores_grad(z, t, st, en, a, b, g, stream=s)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        x, tt = logits_of(rows, vocab, torch.bfloat16, 100 + seed)
        z.copy_(x)
        t.copy_(tt)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (lp, st, en, ai, al, g)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (lp, st, en, ai, al, g)))
        want = ref.scores(x.double(), tt, 1.0, 5)
        assert torch.equal(ai.cpu().long(), want["alt_ids"])


def test_another_stream(gpu):
    z, t = logits_of(10, 8449, torch.bfloat16, 29)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    check(z, t, 5, stream=s.cuda_stream)
