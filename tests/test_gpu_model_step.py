"""The calls of a serving step together: plan, append, attention, adjusted logits, scores; and the gradient back through them."""

import math

import pytest

torch = pytest.importorskip("torch")
from cache_reference import U32, UNIT, adjusted, rotate  # noqa: E402
from paper_2607_29678_amd import (adjust_logits, adjust_logits_grad, cache_append, cache_attention,  # noqa: E402
                                  cache_attention_workspace, step_plan, token_scores, token_scores_grad, token_scores_workspace)

pytestmark = pytest.mark.gpu
PAGE, HEADS, KV, DIM, VOCAB, ALT = 16, 8, 2, 64, 1_281, 3
I32 = dict(dtype=torch.int32, device="cuda")
BF = torch.bfloat16


class Server:
    """A model of one attention layer: embeddings are queries, keys and values, logits are the attention's output times a matrix."""

    def __init__(self, requests, seed=0, pages=200, width=40, room=400):
        g = torch.Generator().manual_seed(seed)
        new = lambda *s: torch.randn(*s, generator=g).to(BF).cuda()  # noqa: E731
        self.embedding, self.head = new(VOCAB, (HEADS + 2 * KV) * DIM), new(HEADS * DIM, VOCAB) * 0.3
        self.frequencies = (10_000.0 ** (-torch.arange(DIM // 2) / (DIM // 2))).float().cuda()
        self.keys, self.values = (torch.full((pages, PAGE, KV, DIM), math.nan, dtype=BF, device="cuda") for _ in range(2))
        self.tables = torch.full((requests, width), -1, **I32)
        self.free, self.count = torch.arange(pages, **I32), torch.tensor([pages], device="cuda")
        self.cached, self.held = torch.zeros(requests, **I32), torch.zeros(requests, **I32)
        self.n, self.room = requests, room
        i64 = dict(dtype=torch.int64, device="cuda")
        self.s = dict(offsets=torch.empty(requests + 1, **I32), lengths=torch.empty(requests, **I32), pages=torch.empty(requests, **I32),
                      slots=torch.empty(room, **i64), positions=torch.empty(room, **I32), requests=torch.empty(room, **I32),
                      targets=torch.empty(room, **I32), result=torch.empty(2, **i64))
        self.ids, self.fresh = torch.zeros(room, **I32), torch.zeros(requests, **I32)
        self.turned, self.out = (torch.zeros(room, HEADS, DIM, dtype=BF, device="cuda") for _ in range(2))
        self.work = torch.empty(cache_attention_workspace(room, requests, HEADS, KV, DIM), dtype=torch.uint8, device="cuda")
        self.texts = [[] for _ in range(requests)]  # what each request's cache holds

    def run(self, window, sinks):
        """Every device call of a step; may be captured."""
        stream, s = torch.cuda.current_stream().cuda_stream, self.s
        step_plan(self.cached, self.fresh, self.tables, self.free, self.count, PAGE, held=self.held, ids=self.ids, stream=stream, **s)
        x = self.embedding[self.ids.long()]
        q, k, v = (part.unflatten(1, (-1, DIM)) for part in x.split((HEADS * DIM, KV * DIM, KV * DIM), 1))
        cache_append(k, v, self.keys, self.values, s["slots"], s["positions"], self.frequencies, queries=q, rotated=self.turned,
                     stream=stream)
        cache_attention(self.turned, self.keys, self.values, self.tables, s["offsets"], s["lengths"], self.out, window=window,
                        sinks=sinks, workspace=self.work, stream=stream)

    def step(self, parts, kept=None, window=0, sinks=0, run=None):
        if kept is not None:
            self.cached.copy_(torch.tensor(kept, dtype=torch.int32))
            self.texts = [t[:k] for t, k in zip(self.texts, kept)]
        ids = [i for p in parts for i in p]
        self.ids[:len(ids)] = torch.tensor(ids, dtype=torch.int32, device="cuda")
        self.fresh.copy_(torch.tensor([len(p) for p in parts], dtype=torch.int32))
        self.texts = [t + list(p) for t, p in zip(self.texts, parts)]
        (run or self.run)(window, sinks)
        assert int(self.s["result"][0]) == len(ids)
        self.cached.copy_(self.s["lengths"])
        self.held.copy_(self.s["pages"])
        self.count.copy_(self.s["result"][1:])
        return len(ids)

    def dense(self, r, window, sinks):
        """float64 attention of all tokens of a request, from its text alone, and a bound of the error of the cached one."""
        x = self.embedding.cpu()[torch.tensor(self.texts[r], dtype=torch.int64)].double()
        n, u = len(x), UNIT[BF]
        q, k, v = (part.unflatten(1, (-1, DIM)) for part in x.split((HEADS * DIM, KV * DIM, KV * DIM), 1))
        p = torch.arange(n)
        q, k = (rotate(y, p, self.frequencies.cpu(), False)[0] for y in (q, k))
        k, v = (y.repeat_interleave(HEADS // KV, 1) for y in (k, v))
        z = torch.einsum("ihd,jhd->hij", q, k) * DIM ** -0.5
        size = torch.einsum("ihd,jhd->hij", q.abs(), k.abs()).amax(2, keepdim=True) * DIM ** -0.5
        seen = p[None] <= p[:, None]
        if window:
            seen &= (p[None] > p[:, None] - window) | (p[None] < sinks)
        w = torch.softmax(z.masked_fill(~seen, -math.inf), 2)
        y, most = torch.einsum("hij,jhd->ihd", w, v), torch.einsum("hij,jhd->ihd", w, v.abs())
        # queries and keys are rounded once each (2 u of a score's terms), weights and results too
        off = (2 * (2 * u + (DIM + 4) * U32) * size[..., 0].t()[..., None] * (1 + u) + 2 * u + n * U32) * most + u * y.abs()
        return y, off

    def check(self, parts, window=0, sinks=0):
        at = 0
        for r, p in enumerate(parts):
            if p:
                want, off = self.dense(r, window, sinks)
                got = self.out[at:at + len(p)].double().cpu()
                assert bool(((got - want[-len(p):]).abs() <= off[-len(p):]).all()), (r, float((got - want[-len(p):]).abs().max()))
            at += len(p)


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_steps(gpu, window, sinks):
    """Prompts, single tokens, a repair that gives tokens back, and requests that rest."""
    g = torch.Generator().manual_seed(3)
    text = lambda n: torch.randint(0, VOCAB, (n,), generator=g).tolist()  # noqa: E731
    s = Server(5)
    for parts, kept in (([text(70), text(1), text(16), text(33), []], None), ([text(1) for _ in range(5)], None),
                        ([text(1), [], text(5), text(1), text(120)], None), ([text(3), text(2), [], text(9), text(1)], [60, 1, 22, 30, 100]),
                        ([text(1) for _ in range(5)], None)):
        s.step(parts, kept, window, sinks)
        s.check(parts, window, sinks)


def test_captured_steps(gpu):
    """One graph of the device calls serves steps of other lengths, with eager work between its replays."""
    g = torch.Generator().manual_seed(4)
    s = Server(4, room=24)
    parts = [[1], [2], [3], [4]]
    s.step(parts)
    s.check(parts)
    torch.cuda.synchronize()
    # captured on the state of a step that brings nothing
    s.fresh.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(10, 2)
    for sizes in ((1, 1, 1, 1), (5, 0, 1, 18), (1, 1, 1, 1), (0, 9, 0, 0), (1, 0, 1, 1)):
        parts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in sizes]
        s.step(parts, window=10, sinks=2, run=lambda *_: graph.replay())
        s.check(parts, 10, 2)


def test_answers_with_penalties_and_masks(gpu):
    """Greedy answers under a mask and penalties: each is the best token of the plain adjusted logits, up to their rounding."""
    s = Server(3)
    parts = [[5, 9, 9, 700], [11], [3] * 20]
    masks = torch.full((1, (VOCAB + 31) // 32), 0x0F0F0F0F, **I32)
    allowed = torch.tensor([(j % 8) < 4 for j in range(VOCAB)])
    mask_rows = torch.tensor([0, -1, 0], **I32)
    rep, pres, freq = (torch.full((3,), x, device="cuda") for x in (1.3, 0.4, 0.2))
    need = token_scores_workspace(3, VOCAB, ALT)
    room = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    for _ in range(6):
        s.step(parts)
        last = (s.s["offsets"][1:] - 1).long()
        logits = (s.out[last].flatten(1).float() @ s.head.float()).to(BF)
        history = torch.tensor([i for t in s.texts for i in t], **I32)
        ends = torch.tensor([0] + [len(t) for t in s.texts], device="cuda").cumsum(0)
        out = torch.empty_like(logits)
        adjust_logits(logits, out, history, ends, rep, pres, freq, masks=masks, mask_rows=mask_rows)
        ids, lp = torch.empty(3, ALT, **I32), torch.empty(3, ALT, device="cuda")
        token_scores(out, None, alt_ids=ids, alt_logprobs=lp, workspace=room)
        want, size = adjusted(logits.double().cpu(), s.texts, rep, pres, freq, None, [allowed, None, allowed])
        for r in range(3):
            best = ids[r, 0].item()
            assert r == 1 or allowed[best]
            assert float(want[r, best]) >= float(want[r].max()) - 2 * 2.0 ** -7 * float(size[r].max())
        parts = [[i] for i in ids[:, 0].tolist()]


def test_gradient_through_both(gpu):
    """The gradient of given tokens' log probabilities and entropies back to the raw logits, against automatic differentiation."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(6, VOCAB, generator=g) * 2
    texts = [torch.randint(0, 40, (30,), generator=g).tolist() for _ in range(6)]
    rep = torch.rand(6, generator=g) + 0.7
    allowed = torch.rand(VOCAB, generator=g) < 0.5
    targets = [int(i) for i in torch.nonzero(allowed)[:6, 0]]
    a, b = torch.randn(6, generator=g), torch.randn(6, generator=g)
    z = x.double().requires_grad_()
    hit = torch.zeros(6, VOCAB, dtype=torch.bool)
    for r, t in enumerate(texts):
        hit[r, t] = True
    y = torch.where(hit, torch.where(z > 0, z / rep[:, None].double(), z * rep[:, None].double()), z).masked_fill(~allowed, -math.inf)
    logp = torch.log_softmax(y, 1)
    p = logp.exp()
    entropy = -(p * torch.where(allowed, logp, torch.zeros_like(logp))).sum(1)
    (a.double() * logp[torch.arange(6), targets] + b.double() * entropy).sum().backward()

    bits = torch.zeros(((VOCAB + 31) // 32) * 32, dtype=torch.int64)
    bits[:VOCAB] = allowed.long()
    words = (bits.view(-1, 32) << torch.arange(32)).sum(1)
    masks = torch.where(words >= 2**31, words - 2**32, words).int()[None].cuda()
    history = torch.tensor([i for t in texts for i in t], **I32)
    ends = torch.arange(7, device="cuda") * 30
    common = dict(masks=masks, mask_rows=torch.zeros(6, **I32))
    logits, out, t = x.cuda(), torch.empty(6, VOCAB, device="cuda"), torch.tensor(targets, **I32)
    adjust_logits(logits, out, history, ends, rep.cuda(), **common)
    lp, stats, h = torch.empty(6, device="cuda"), torch.empty(6, 2, device="cuda"), torch.empty(6, device="cuda")
    room = torch.empty(max(token_scores_workspace(6, VOCAB), 1), dtype=torch.uint8, device="cuda")
    token_scores(out, t, lp, stats, h, workspace=room)
    token_scores_grad(out, t, stats, h, a.cuda(), b.cuda(), out)  # in place, and the next call too
    adjust_logits_grad(logits, out, out, history, ends, rep.cuda(), **common)
    # sums of 1,281 terms, exponents of at most 32 and the statistics' roundings, on terms of at most (|a| + 14 |b|) * 1.7
    size = ((a.abs() + 14 * b.abs()) * 1.7)[:, None].double()
    assert bool(((out.double().cpu() - z.grad).abs() <= size * U32 * (4 * 32 + VOCAB / 256 + 64)).all())
