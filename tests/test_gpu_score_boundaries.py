"""Token scores on both sides of every rule that chooses a kernel: rows in parts or whole, a block or a wave a row.

The workspace has exactly the size asked for, and what lies behind it and behind the outputs stays as it was.
"""

import math

import pytest

torch = pytest.importorskip("torch")
import model_reference as ref  # noqa: E402
import paper_2607_29678_amd as tt  # noqa: E402

pytestmark = pytest.mark.gpu
GUARD = 512


def guarded(n, dtype, fill):
    """(the n entries to use, the whole buffer): GUARD entries of `fill` stand behind them."""
    whole = torch.full((n + GUARD,), fill, dtype=dtype, device="cuda")
    return whole[:n], whole


def check(rows, vocab, kind, n_alt, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed + rows + vocab + n_alt)
    z = (torch.randn(rows, vocab, generator=gen, device="cuda") * 2.5).to(kind)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    t[0], t[rows // 2], t[-1] = 0, -1, vocab - 1
    z[rows // 3, : vocab - 7] = -math.inf
    need = tt.token_scores_workspace(rows, vocab, n_alt)
    room, room_all = guarded(need, torch.uint8, 0xA5)
    lp, lp_all = guarded(rows, torch.float32, 77.0)
    st, st_all = guarded(2 * rows, torch.float32, 77.0)
    en, en_all = guarded(rows, torch.float32, 77.0)
    ids, ids_all = guarded(rows * n_alt, torch.int32, -77)
    al, al_all = guarded(rows * n_alt, torch.float32, 77.0)
    alt = dict(alt_ids=ids.view(rows, n_alt), alt_logprobs=al.view(rows, n_alt)) if n_alt else {}
    tt.token_scores(z, t, lp, st.view(rows, 2), en, workspace=room if need else None, **alt)
    torch.cuda.synchronize()
    for whole, n, fill in ((room_all, need, 0xA5), (lp_all, rows, 77), (st_all, 2 * rows, 77), (en_all, rows, 77),
                           (ids_all, rows * n_alt, -77), (al_all, rows * n_alt, 77)):
        assert bool((whole[n:] == fill).all())
    d = z.double()
    m = d.amax(1)
    lse = torch.logsumexp(d, 1)
    logp = d - lse[:, None]
    tol = ref.score_error(vocab, float((m - d[torch.isfinite(d)].min()).max()))
    want = torch.where(t < 0, torch.zeros_like(m), logp.gather(1, t.clamp(min=0).long()[:, None])[:, 0])
    ref.close(lp, want, tol + 4 * ref.U32 * want.abs().nan_to_num(posinf=0))
    assert torch.equal(st.view(rows, 2)[:, 0].double(), m)
    ref.close(st.view(rows, 2)[:, 1], lse - m, tol)
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    ref.close(en, entropy, 2 * tol * (1 + math.log(vocab)))
    if n_alt:
        # one key an entry: by value, the lowest index first among equals
        bits = z.float().view(torch.int32)
        key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32) + (0x7FFFFFFF - torch.arange(vocab, device="cuda"))
        best = 0x7FFFFFFF - (torch.topk(key, n_alt, dim=1).values & 0xFFFFFFFF)
        value = logp.gather(1, best)
        assert torch.equal(ids.view(rows, n_alt).long(), torch.where(value == -math.inf, torch.full_like(best, -1), best))
        ref.close(al.view(rows, n_alt), value, tol + 4 * ref.U32 * value.abs().nan_to_num(posinf=0))


@pytest.mark.parametrize("rows", [256, 257])
def test_most_rows_in_parts(gpu, rows):
    check(rows, 120_001, torch.bfloat16, 0)


@pytest.mark.parametrize("n_alt", [1, 64])
@pytest.mark.parametrize("rows", [512, 513])
def test_most_rows_in_parts_with_alternatives(gpu, rows, n_alt):
    check(rows, 130_001, torch.bfloat16, n_alt)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_alt", [0, 20])
@pytest.mark.parametrize("vocab", [24_575, 24_576, 40_959, 40_960])
def test_shortest_rows_in_parts(gpu, vocab, n_alt, kind):
    check(8, vocab, kind, n_alt)
    check(101, vocab * 101 // 100 + (vocab * 101 % 100 > 0), kind, n_alt)


@pytest.mark.parametrize("n_alt", [0, 64])
@pytest.mark.parametrize("vocab", [16_384, 16_385])
@pytest.mark.parametrize("rows", [2_047, 2_048])
def test_rows_of_a_wave_and_of_a_block(gpu, rows, vocab, n_alt):
    check(rows, vocab, torch.bfloat16, n_alt)


@pytest.mark.parametrize("kind", [torch.float32, torch.float16])
@pytest.mark.parametrize("past", [0, 1])
def test_gradient_of_a_wave_and_of_a_block(gpu, kind, past):
    """The longest row that one wave takes (1,024 or 2,048 entries), and one entry more."""
    vocab = 64 * 4 * 16 // torch.empty(0, dtype=kind).element_size() + past
    rows = 5
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = torch.randn(rows, vocab, generator=gen, device="cuda").to(kind)
    t = torch.tensor([0, vocab - 1, -1, 7, vocab // 2], dtype=torch.int32, device="cuda")
    a = torch.linspace(-1, 1, rows, device="cuda")
    lse, m = torch.logsumexp(z.double(), 1), z.double().amax(1)
    g, whole = guarded(rows * vocab, kind, 9.0)
    tt.token_scores_grad(z, t, torch.stack([m, lse - m], 1).float(), None, a, None, g.view(rows, vocab))
    torch.cuda.synchronize()
    assert bool((whole[rows * vocab:] == 9).all())
    want, size = ref.logits_grad(z.double(), t, a.double(), torch.zeros(rows, dtype=torch.float64, device="cuda"))
    unit, least = ref.ROUNDING[kind]
    ref.close(g.view(rows, vocab), want, size * 200 * ref.U32 + unit * want.abs() + least)
