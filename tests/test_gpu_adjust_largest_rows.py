"""``tt_adjust_logits`` and its gradient at the longest rows that the calls take, 2^31 - 1 columns: their ends are like any."""

import math

import pytest

torch = pytest.importorskip("torch")
from paper_2607_29678_amd import adjust_logits, adjust_logits_grad  # noqa: E402

pytestmark = pytest.mark.gpu
PIECE = 1 << 27


def row(vocab, lead, seed):
    """f16 [1, vocab] of whole numbers from -50 to 50, `lead` elements behind an aligned place, all else NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    block = torch.randint(-50, 51, (PIECE,), generator=g, device="cuda").half()
    store = torch.full((vocab + 16,), math.nan, dtype=torch.float16, device="cuda")
    for part in store[lead:lead + vocab].split(PIECE):
        part.copy_(block[:len(part)])
    return store, store[lead:lead + vocab].view(1, vocab)


@pytest.mark.parametrize("vocab,lead", [(2**31 - 1, 0), (2**31 - 1, 3), (2**31 - 200, 0)])
def test_ends_of_the_longest_rows(gpu, vocab, lead):
    stream = torch.cuda.current_stream().cuda_stream
    _, x = row(vocab, lead, 1)
    named = [0, 7, 4_096, 2**30 + 5, vocab - 9, vocab - 8, vocab - 2, vocab - 1]
    history = torch.tensor(named + [vocab, -1], dtype=torch.int32, device="cuda")
    ends = torch.tensor([0, len(history)], device="cuda")
    two, one = (torch.tensor([y], device="cuda") for y in (2.0, 1.0))
    biases = torch.tensor([3, vocab - 1], dtype=torch.int32, device="cuda")
    values, bias_ends = torch.tensor([100.0, 200.0], device="cuda"), torch.tensor([0, 2], device="cuda")
    masks = torch.full((1, (vocab + 31) // 32), -1, dtype=torch.int32, device="cuda")
    barred = [5, 2**30 + 6, vocab - 8, vocab - 3]
    for j in barred:
        masks[0, j // 32] &= ~(1 << j % 32) if j % 32 < 31 else 2**31 - 1
    mask_rows = torch.zeros(1, dtype=torch.int32, device="cuda")

    # halves, doubles and whole numbers below 2^11 are exact in f16
    want = {j: (v / 2 if v > 0 else 2 * v) - 1 for j in named for v in [float(x[0, j])]}
    want[3] = float(x[0, 3]) + 100
    want[vocab - 1] += 200
    want.update({j: -math.inf for j in barred})
    store, out = row(vocab, lead, 2)
    adjust_logits(x, out, history, ends, repetition=two, presence=one, bias_ids=biases, bias_values=values, bias_offsets=bias_ends,
                  masks=masks, mask_rows=mask_rows, stream=stream)
    torch.cuda.synchronize()
    assert {j: float(out[0, j]) for j in want} == want
    for j in want:
        out[0, j] = x[0, j]
    assert all(torch.equal(a, b) for a, b in zip(out[0].split(PIECE), x[0].split(PIECE)))
    assert bool(store[:lead].isnan().all()) and bool(store[lead + vocab:].isnan().all())

    # the gradient, in place
    want = {j: v / 2 if float(x[0, j]) > 0 else 2 * v for j in named for v in [float(out[0, j]) + 1]}
    want.update({j: 0.0 for j in barred})
    for part in out[0].split(PIECE):
        part.add_(1)
    adjust_logits_grad(x, out, out, history, ends, repetition=two, masks=masks, mask_rows=mask_rows, stream=stream)
    torch.cuda.synchronize()
    assert {j: float(out[0, j]) for j in want} == want
    for j in want:
        out[0, j] = x[0, j] + 1
    assert all(torch.equal(a, b + 1) for a, b in zip(out[0].split(PIECE), x[0].split(PIECE)))
    assert bool(store[:lead].isnan().all()) and bool(store[lead + vocab:].isnan().all())
