"""``tt_adjust_logits`` and its gradient against plain 64-bit forms: lists, masks, types, strides, special values, differences."""

import math
import random

import pytest

torch = pytest.importorskip("torch")
from cache_reference import adjusted, adjusted_tolerance  # noqa: E402
from model_reference import close  # noqa: E402
from paper_2607_29678_amd import adjust_logits, adjust_logits_grad, token_scores, token_scores_workspace  # noqa: E402

pytestmark = pytest.mark.gpu
F, BF, H = torch.float32, torch.bfloat16, torch.float16


def flat(lists, dtype, value=lambda x: x):
    ends = [0]
    for x in lists:
        ends.append(ends[-1] + len(x))
    return (torch.tensor([value(x) for row in lists for x in row], dtype=dtype, device="cuda"),
            torch.tensor(ends, dtype=torch.int64, device="cuda"))


def words_of(masks, vocab, spare=0):
    n = (vocab + 31) // 32 + spare
    out = torch.zeros(len(masks), n, dtype=torch.int64)
    for m, allowed in enumerate(masks):
        bits = torch.zeros(n * 32, dtype=torch.int64)
        bits[:vocab] = allowed.long()
        bits[vocab:] = 1
        out[m] = (bits.view(n, 32) << torch.arange(32)).sum(1)
    return torch.where(out >= 2**31, out - 2**32, out).int().cuda()


class Case:
    def __init__(self, rows, vocab, dtype, seed=0, history=30, biases=0, masks=0, lead=0, pitch=0, spare=0):
        rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
        self.rows, self.vocab, self.dtype = rows, vocab, dtype
        pitch = vocab + pitch
        self.store = (torch.randn(lead + rows * pitch, generator=g) * 3).to(dtype).cuda()
        self.logits = self.store[lead:].view(rows, pitch)[:, :vocab]
        self.history = [[rng.choice((rng.randrange(-3, vocab + 3), rng.randrange(min(vocab, 9)))) for _ in range(rng.randint(0, 2 * history))]
                        for _ in range(rows)]
        self.biases = [[(rng.randrange(-2, vocab + 2), rng.gauss(0, 4)) for _ in range(rng.randint(0, 2 * biases))]
                       for _ in range(rows)] if biases else None
        f = lambda a, b: torch.rand(rows, generator=g) * (b - a) + a  # noqa: E731
        self.repetition, self.presence, self.frequency = f(0.7, 1.6), f(-1, 1), f(-0.5, 0.5)
        self.masks = [torch.rand(vocab, generator=g) < p for p in (0.5, 0.01, 0.99, 0.0)[:masks]]
        self.mask_rows = [rng.randrange(-1, masks) for _ in range(rows)] if masks else None
        self.args = {}
        if history:
            self.args["history"], self.args["history_offsets"] = flat(self.history, torch.int32)
            self.args.update(repetition=self.repetition.cuda(), presence=self.presence.cuda(), frequency=self.frequency.cuda())
        else:
            self.history = None
        if biases:
            self.args["bias_ids"], self.args["bias_offsets"] = flat(self.biases, torch.int32, lambda x: x[0])
            values, _ = flat(self.biases, torch.float32, lambda x: x[1])
            self.args["bias_values"] = values
            v = values.tolist()
            self.biases = [[(j, v.pop(0)) for j, _ in row] for row in self.biases]  # (as rounded to 32 bits)
        if masks:
            self.args["masks"] = words_of(self.masks, vocab, spare)
            self.args["mask_rows"] = torch.tensor(self.mask_rows, dtype=torch.int32, device="cuda")

    def want(self, grad=None):
        allowed = None
        if self.mask_rows:
            allowed = [None if m < 0 else "bad" if m >= len(self.masks) else self.masks[m] for m in self.mask_rows]
        p = self.args
        return adjusted(self.logits.double().cpu(), self.history, self.repetition if "repetition" in p else None,
                        self.presence if "presence" in p else None, self.frequency if "frequency" in p else None, self.biases,
                        allowed, grad)

    def gradient_args(self):
        return {k: v for k, v in self.args.items() if k in ("history", "history_offsets", "repetition", "masks", "mask_rows")}


def check(c, out=None):
    out = torch.full((c.rows, c.vocab), 5.0, dtype=c.dtype, device="cuda") if out is None else out
    want, size = c.want()
    adjust_logits(c.logits, out, stream=torch.cuda.current_stream().cuda_stream, **c.args)
    torch.cuda.synchronize()
    close(out, want, adjusted_tolerance(want, size.nan_to_num(0, 0, 0), c.dtype))
    return out


def check_grad(c, seed=1, in_place=False):
    g = torch.randn(c.rows, c.vocab, generator=torch.Generator().manual_seed(seed)).to(c.dtype).cuda()
    want, size = c.want(g.double().cpu())
    out = g if in_place else torch.full_like(g, 5.0)
    adjust_logits_grad(c.logits, g, out, stream=torch.cuda.current_stream().cuda_stream, **c.gradient_args())
    torch.cuda.synchronize()
    close(out, want, adjusted_tolerance(want, size, c.dtype))


SHAPES = [(1, 1), (3, 7), (5, 31), (2, 33), (7, 1_281), (3, 8_449), (2, 50_257), (1, 100_257), (65, 4_096), (2, 8_192), (3, 4_097),
          (600, 130)]


@pytest.mark.parametrize("dtype", [F, BF, H])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_everything(gpu, rows, vocab, dtype):
    c = Case(rows, vocab, dtype, seed=vocab, history=40, biases=10, masks=4)
    check(c)
    check_grad(c)


@pytest.mark.parametrize("dtype", [F, BF, H])
@pytest.mark.parametrize("history,biases,masks", [(0, 0, 0), (20, 0, 0), (0, 12, 0), (0, 0, 3), (20, 12, 0), (20, 0, 3), (0, 12, 3)])
def test_parts(gpu, history, biases, masks, dtype):
    c = Case(6, 5_003, dtype, history=history, biases=biases, masks=masks)
    check(c)
    check_grad(c)
    for name in ("repetition", "presence", "frequency"):
        c = Case(6, 5_003, dtype, history=history, biases=biases, masks=masks)
        c.args.pop(name, None)
        check(c)
        check_grad(c)


@pytest.mark.parametrize("dtype", [F, BF, H])
@pytest.mark.parametrize("lead,pitch", [(1, 0), (0, 1), (3, 5), (8, 8), (4, 31)])
def test_strides(gpu, lead, pitch, dtype):
    c = Case(5, 2_001, dtype, biases=5, masks=2, lead=lead, pitch=pitch, spare=3)
    check(c)
    check_grad(c)
    store = torch.full((lead + 5 * (2_001 + 7),), 5.0, dtype=dtype, device="cuda")
    check(c, store[lead:].view(5, -1)[:, :2_001])
    assert bool((store[:lead] == 5).all()) and bool((store[lead:].view(5, -1)[:, 2_001:] == 5).all())


@pytest.mark.parametrize("dtype", [F, BF, H])
def test_in_place(gpu, dtype):
    c = Case(4, 9_001, dtype, biases=5, masks=3, pitch=3)
    before = c.store.clone()
    check(c, c.logits)
    rest = torch.ones_like(c.store, dtype=torch.bool).view(4, -1)
    rest[:, :9_001] = False
    assert torch.equal(c.store[rest.view(-1)], before[rest.view(-1)])
    check_grad(Case(4, 9_001, dtype, masks=3), in_place=True)


@pytest.mark.parametrize("dtype", [F, BF, H])
@pytest.mark.parametrize("over", range(-9, 10))
def test_ends_of_runs(gpu, dtype, over):
    """Lists that name the columns around 4,096 and 8,192, where a block's run of columns ends, and a row's first and last ones."""
    for vocab in (4_096 + over, 8_192 + over):
        c = Case(4, vocab, dtype, biases=2, masks=1, pitch=1)
        ids = list(range(4_080, min(vocab, 4_110))) + list(range(vocab - 20, vocab)) + list(range(10))
        c.history = [ids] * 4
        c.args["history"], c.args["history_offsets"] = flat(c.history, torch.int32)
        c.biases = [[(j, float(j % 7)) for j in ids[::2]]] * 4
        c.args["bias_ids"], c.args["bias_offsets"] = flat(c.biases, torch.int32, lambda x: x[0])
        c.args["bias_values"], _ = flat(c.biases, torch.float32, lambda x: x[1])
        for lead in range(2):  # outputs of other alignments
            store = torch.zeros(lead + 4 * (vocab + 3), dtype=dtype, device="cuda")
            check(c, store[lead:].view(4, -1)[:, :vocab])
        check_grad(c)


def test_long_histories(gpu):
    """A token that stands more than 2^16 times, and a list longer than its neighbours."""
    c = Case(3, 700, F, history=5)
    c.history = [[5] * 70_000 + [6] * 65_536 + [7], [], list(range(700)) * 3]
    c.args["history"], c.args["history_offsets"] = flat(c.history, torch.int32)
    check(c)


def test_the_last_bias_of_a_token_counts(gpu):
    c = Case(2, 500, F, history=0, biases=3)
    c.biases = [[(7, 1.0), (9, 4.0), (7, -2.0)], [(3, 5.0)] * 400 + [(3, 0.5)]]
    c.args["bias_ids"], c.args["bias_offsets"] = flat(c.biases, torch.int32, lambda x: x[0])
    c.args["bias_values"], _ = flat(c.biases, torch.float32, lambda x: x[1])
    out = check(c)
    x = c.logits
    assert torch.equal(out[0, 7], x[0, 7] - 2) and torch.equal(out[0, 9], x[0, 9] + 4) and torch.equal(out[1, 3], x[1, 3] + 0.5)


def test_special_values(gpu):
    for dtype in (F, BF, H):
        c = Case(3, 300, dtype, history=10, masks=2)
        c.mask_rows = [0, -1, 1]
        c.args["mask_rows"] = torch.tensor(c.mask_rows, dtype=torch.int32, device="cuda")
        c.history = [[1, 2, 3, 4]] * 3
        c.args["history"], c.args["history_offsets"] = flat(c.history, torch.int32)
        c.logits[:, 1], c.logits[:, 2], c.logits[:, 3] = math.nan, math.inf, -math.inf
        c.logits[:, 5:200] = math.nan  # what the masks do not allow does not matter
        c.logits[:, 200] = torch.finfo(dtype).min
        out = check(c)
        assert not bool(torch.isnan(out[0, ~c.masks[0].cuda()]).any())


def test_masks_that_leave_nothing(gpu):
    c = Case(3, 1_000, BF, masks=4)
    c.mask_rows = [3, 3, -1]
    c.args["mask_rows"] = torch.tensor(c.mask_rows, dtype=torch.int32, device="cuda")
    out = check(c)
    lp, h = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    need = token_scores_workspace(3, 1_000)
    token_scores(out, torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), lp, entropy=h,
                 workspace=torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"))
    assert lp[:2].tolist() == [-math.inf] * 2 and h[:2].tolist() == [0, 0] and math.isfinite(float(lp[2]))


def test_numbers_that_are_no_mask(gpu):
    c = Case(4, 1_000, BF, masks=2)
    c.mask_rows = [2, 0, 2**31 - 1, -2**31]
    c.args["mask_rows"] = torch.tensor(c.mask_rows, dtype=torch.int32, device="cuda")
    check(c)
    check_grad(c)


def test_offsets_outside_the_lists(gpu):
    c = Case(3, 500, F, history=10, biases=5)
    n, m = len(c.args["history"]), len(c.args["bias_ids"])
    whole, pairs = c.args["history"].tolist(), list(zip(c.args["bias_ids"].tolist(), c.args["bias_values"].tolist()))
    for ends, want in (([0, n, 2 * n, 2**62], (whole, [], [])), ([-5, 3, 1, n], (whole[:3], [], whole[1:])),
                       ([2**62, -2**62, 4, 4], ([], whole[:4], []))):
        c.args["history_offsets"] = torch.tensor(ends, device="cuda")
        c.history = list(want)
        b = [min(max(e, 0), m) for e in ends]
        c.args["bias_offsets"] = torch.tensor(ends, device="cuda")
        c.biases = [pairs[x:max(x, y)] for x, y in zip(b[:-1], b[1:])]
        check(c)


def test_nothing(gpu):
    z = torch.zeros(0, 50, device="cuda")
    adjust_logits(z, z.clone())
    adjust_logits_grad(z, z.clone(), z.clone())
    x = torch.randn(3, 50, device="cuda")
    none, ends = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    out = torch.empty_like(x)
    adjust_logits(x, out, none, ends, repetition=torch.full((3,), 2.0, device="cuda"), bias_ids=none, bias_offsets=ends,
                  bias_values=torch.zeros(0, device="cuda"))
    assert torch.equal(out, x)


def test_gradient_against_differences(gpu):
    """In 32 bits at steps of 2^-6 the result changes by exactly its slope, but for roundings of values below 16."""
    c = Case(3, 400, F, history=60, masks=2)
    c.logits.copy_(torch.where(c.logits.abs() < 0.1, torch.full_like(c.logits, 0.5), c.logits))  # (no step crosses 0)
    step = 2.0 ** -6
    ones, slope = torch.ones(3, 400, device="cuda"), torch.empty(3, 400, device="cuda")
    adjust_logits_grad(c.logits, ones, slope, **c.gradient_args())
    up, down = torch.empty_like(ones), torch.empty_like(ones)
    adjust_logits(c.logits + step, up, **c.args)
    adjust_logits(c.logits - step, down, **c.args)
    got = torch.where(torch.isinf(up), torch.zeros_like(up), (up - down) / (2 * step))
    # two results, each of at most six roundings (the sum with the step among them) of values below 128
    assert float(up[torch.isfinite(up)].abs().max()) < 128
    close(slope, got.double().cpu(), 2 * 6 * 128 * 2.0 ** -24 / (2 * step))


def test_graph_replays_on_new_contents(gpu):
    c = Case(4, 9_001, BF, biases=5, masks=3)
    out, grad = torch.empty(4, 9_001, dtype=BF, device="cuda"), torch.randn(4, 9_001, device="cuda").to(BF)
    grad_in = torch.empty_like(grad)
    check(c)
    check_grad(c)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        stream = torch.cuda.current_stream().cuda_stream
        adjust_logits(c.logits, out, stream=stream, **c.args)
        adjust_logits_grad(c.logits, grad, grad_in, stream=stream, **c.gradient_args())
    for k in range(4):
        c.logits.neg_()
        c.args["history"].copy_(torch.randint(0, 9_001, c.args["history"].shape, device="cuda"))
        c.args["mask_rows"].copy_(torch.tensor([k - 1, 2, 0, -1], dtype=torch.int32))
        g.replay()
        want, want_grad = torch.empty_like(out), torch.empty_like(grad)
        adjust_logits(c.logits, want, **c.args)
        adjust_logits_grad(c.logits, grad, want_grad, **c.gradient_args())
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(grad_in, want_grad)


def test_rows_past_32_bits(gpu):
    """Elements behind the 2^31st."""
    rows, vocab = 43_000, 50_257
    x = torch.zeros(rows, vocab, dtype=BF, device="cuda")
    x[-1] = 1.0
    ends = torch.zeros(rows + 1, dtype=torch.int64, device="cuda")
    ends[-1] = 2
    history = torch.tensor([50_256, 3], dtype=torch.int32, device="cuda")
    rep = torch.full((rows,), 2.0, device="cuda")
    adjust_logits(x, x, history, ends, rep)
    last = x[-1].float()
    assert last[3] == 0.5 and last[50_256] == 0.5 and float(last.sum()) == vocab - 1
    assert not bool(x[:-1].any())
