"""The operators on both sides of a model, as performance cases: the plan of a step's tokens, and the scores of given tokens.

``plan``: positions, cache slots, page tables and next-token targets of a serving step, from the
requests' lengths.  ``scores`` and ``scores_grad``: log probabilities of given tokens, entropy and
top alternatives of stored logits, and the gradient.  ``head`` and ``head_grad``: the same scores
from hidden states and the head's weights without stored logits, and both gradients.  Vocabulary
sizes are those of the stored merge tables (1,281, 8,449, 50,257 and 100,257 entries).
"""

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
VOCABS = (1_281, 8_449, 50_257, 100_257)


def listed():
    return [
        # a decode step of a busy server: one new token a request, launch latency counts
        dict(name="plan decode 96", op="plan", requests=96, tokens=96, page=16, context=4_000, held=False),
        # decode and chunked prefill in one step; sessions whose repair gave tokens back hold more pages than they fill
        dict(name="plan mixed 301", op="plan", requests=301, tokens=16_381, page=16, context=6_000, held=True),
        # the documents of a 1M-character batch as one prefill
        dict(name="plan prefill 420k", op="plan", requests=64, tokens=420_000, page=64, context=0, held=False),
        # one decode step of eight requests with five alternatives each
        dict(name="scores decode 8", op="scores", rows=8, vocab=50_257, type="bf16", top=5, padded=False, allowed=1.0),
        # prompt log probabilities of a request, twenty alternatives
        dict(name="scores prompt 2048", op="scores", rows=2_048, vocab=100_257, type="bf16", top=20, padded=False, allowed=1.0),
        # constrained answers: most of a row is -inf; 32-bit logits in rows of padded length
        dict(name="scores masked 501", op="scores", rows=501, vocab=8_449, type="f32", top=8, padded=True, allowed=0.02),
        # policy gradient with an entropy term over stored logits
        dict(name="scores grad 1536", op="scores_grad", rows=1_536, vocab=100_257, type="bf16", padded=False),
        # small vocabulary, many rows
        dict(name="scores grad 4097", op="scores_grad", rows=4_097, vocab=1_281, type="f16", padded=False),
        # the head of a decode step: the weights stream once
        dict(name="head decode 4", op="head", rows=4, width=2_048, vocab=50_257, type="bf16"),
        # the likelihood of a document of 4,001 tokens
        dict(name="head document 4001", op="head", rows=4_001, width=2_048, vocab=100_257, type="bf16"),
        # a small training step on short documents
        dict(name="head grad 640", op="head_grad", rows=640, width=1_024, vocab=50_257, type="f16"),
        # a training step's micro-batch
        dict(name="head grad 2048", op="head_grad", rows=2_048, width=2_048, vocab=100_257, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("plan", "scores", "scores_grad", "head", "head_grad"))
    if op == "plan":
        requests = _log(rng, 1, 4_000)
        kind = rng.choice(("decode", "mixed", "prefill"))
        tokens = requests if kind == "decode" else max(requests, _log(rng, requests + 1, 420_000))
        context = 0 if kind == "prefill" else _log(rng, 16, 8_000)
        return dict(op=op, requests=requests, tokens=tokens, page=rng.choice((8, 16, 16, 24, 32, 64, 128)),
                    context=context, held=bool(context) and rng.random() < 0.5)
    if op in ("scores", "scores_grad"):
        vocab = rng.choice(VOCABS + (_log(rng, 1_000, 100_000),))
        c = dict(op=op, rows=_log(rng, 1, min(8_000, 200_000_000 // vocab)), vocab=vocab,
                 type=rng.choice(("bf16", "bf16", "f16", "f32")), padded=rng.random() < 0.3)
        if c["type"] == "f32":
            c["rows"] = max(1, c["rows"] // 2)
        if op == "scores":
            c.update(top=rng.choice((0, 1, 5, 8, 20, 32)), allowed=rng.choice((1.0, 1.0, 1.0, 0.3, 0.01)))
        return c
    vocab = rng.choice(VOCABS[1:] + (_log(rng, 1_000, 100_000),))
    width = rng.choice((256, 512, 768, 1_000, 1_024, 1_536, 2_048))
    most = (4_001 if op == "head" else 2_048) * 2_048 * 100_257 // (width * vocab)
    return dict(op=op, rows=_log(rng, 1, min(most, 6_000)), width=width, vocab=vocab, type=rng.choice(("bf16", "bf16", "f16")))


def _room(tokens):
    """Entries of the per-token arrays: a step is padded to a multiple of 8, as for a captured graph."""
    return -(-tokens // 8) * 8


def _longest(case):
    """The most new tokens that one request of a step brings."""
    return min(case["tokens"], 6 * case["tokens"] // case["requests"]) + case["tokens"] // case["requests"] + 2


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _prepare_plan(case, seed):
    rng = np.random.RandomState(seed % (1 << 32))
    n, tokens, page = case["requests"], case["tokens"], case["page"]
    most = _longest(case)
    if tokens == n:
        new = np.ones(n, dtype=np.int64)
    else:  # long and short prompts; the rest decode a few tokens
        w = np.where(rng.rand(n) < 0.5, rng.lognormal(0.0, 1.2, n), 0.0)
        w[rng.randint(n)] += 1.0
        new = 1 + np.minimum(np.floor((tokens - n) * w / w.sum()).astype(np.int64), most - 2 - tokens // n)
        rest = tokens - int(new.sum())
        new += rest // n
        new[:rest % n] += 1
    cached = np.zeros(n, dtype=np.int64)
    if case["context"]:
        cached = np.minimum(rng.lognormal(math.log(case["context"]), 0.7, n), 2.0 * case["context"]).astype(np.int64)
    held = -(-cached // page)
    if case["held"]:
        held = held + np.where(rng.rand(n) < 0.3, rng.randint(0, 4, n), 0)
    need = np.maximum(held, -(-(cached + new) // page))
    width = -(-(2 * case["context"] + most) // page) + 4
    take = int((need - held).sum())
    pages = rng.permutation(int(held.sum()) + take + 500).astype(np.int32)
    tables = np.full((n, width), -1, dtype=np.int32)
    at = np.concatenate([[0], np.cumsum(held)])
    col = np.arange(width)
    mine = col[None, :] < held[:, None]
    tables[mine] = pages[:at[-1]]
    free = pages[at[-1]:]
    room = _room(tokens)
    new_i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(
        op="plan", page=page, cached=_dev(cached.astype(np.int32)), new=_dev(new.astype(np.int32)),
        held=_dev(held.astype(np.int32)) if case["held"] else None, tables=_dev(tables), free=_dev(free),
        count=_dev(np.array([len(free)], dtype=np.int64)), ids=_dev(rng.randint(0, 100_257, room).astype(np.int32)),
        offsets=new_i32(n + 1), lengths=new_i32(n), pages=new_i32(n),
        slots=torch.empty(room, dtype=torch.int64, device="cuda"), positions=new_i32(room), requests=new_i32(room),
        targets=new_i32(room), result=torch.empty(2, dtype=torch.int64, device="cuda"))


def _targets(gen, rows, vocab):
    """Given tokens; -1 (none) where a document ends."""
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    ends = torch.rand(rows, generator=gen, device="cuda") < 0.02
    return torch.where(ends, torch.full_like(t, -1), t)


def _gradients(gen, rows):
    """What a policy-gradient loss passes back: advantages for the log probabilities, a small weight for the entropy."""
    g = torch.randn(rows, generator=gen, device="cuda") / rows
    return g, torch.full((rows,), 0.01 / rows, device="cuda")


def _buffers(rows):
    f = lambda *shape: torch.empty(shape, dtype=torch.float32, device="cuda")  # noqa: E731
    return dict(logprobs=f(rows), stats=f(rows, 2), entropy=f(rows))


def _prepare_scores(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, vocab, kind = case["rows"], case["vocab"], TYPES[case["type"]]
    targets = _targets(gen, rows, vocab)
    x = torch.randn(rows, vocab, generator=gen, device="cuda") * 2.5
    lift = torch.rand(rows, generator=gen, device="cuda") * 12 + 2
    liked = torch.where(targets < 0, torch.zeros_like(targets), targets).long()
    x[torch.arange(rows, device="cuda"), liked] += lift  # the model mostly expects the given token
    if case.get("allowed", 1.0) < 1:
        banned = torch.rand(rows, vocab, generator=gen, device="cuda") >= case["allowed"]
        banned[torch.arange(rows, device="cuda"), liked] = False
        x.masked_fill_(banned, -math.inf)
        del banned
    pitch = -(-vocab // 64) * 64 if case["padded"] else vocab
    logits = torch.zeros(rows, pitch, dtype=kind, device="cuda")[:, :vocab]
    logits.copy_(x)
    del x
    state = dict(op=case["op"], vocab=vocab, logits=logits, targets=targets, **_buffers(rows))
    if case["op"] == "scores":
        top = case["top"]
        state.update(top=top, work=torch.empty(_scores_room(rows, vocab, top), dtype=torch.uint8, device="cuda"),
                     alt_ids=torch.empty(rows, top, dtype=torch.int32, device="cuda"),
                     alt_logprobs=torch.empty(rows, top, dtype=torch.float32, device="cuda"))
    else:
        state["g_logprobs"], state["g_entropy"] = _gradients(gen, rows)
        state["stats"], state["entropy"] = _statistics(logits.float())
        state["g_logits"] = torch.empty_like(logits, memory_format=torch.contiguous_format)
    return state


def _scores_room(rows, vocab, top):
    """Workspace of a scores call, with room to spare."""
    return 65_536 + 32_768 * (8 + 8 * top)


def _statistics(x):
    """What the forward pass leaves for the backward one: the largest logit, the logarithm of the sum, the entropy."""
    m = x.amax(1, keepdim=True)
    e = (x - m).exp_()
    s = e.sum(1, keepdim=True)
    h = s.log() - (e * (x - m)).nan_to_num_(0.0).sum(1, keepdim=True) / s
    return torch.cat([m, s.log()], 1), h[:, 0].contiguous()


def _prepare_head(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, width, vocab, kind = case["rows"], case["width"], case["vocab"], TYPES[case["type"]]
    targets = _targets(gen, rows, vocab)
    weight = (torch.randn(vocab, width, generator=gen, device="cuda") * (2.5 / math.sqrt(width))).to(kind)
    hidden = torch.randn(rows, width, generator=gen, device="cuda")
    lift = torch.rand(rows, 1, generator=gen, device="cuda") * 12 + 2
    hidden += lift / 6.25 * weight[targets.clamp(min=0).long()].float()  # |a row of the weights|^2 is about 6.25
    hidden = hidden.to(kind)
    state = dict(op=case["op"], hidden=hidden, weight=weight, targets=targets, **_buffers(rows))
    if case["op"] == "head_grad":
        state["g_logprobs"], state["g_entropy"] = _gradients(gen, rows)
        state["stats"], state["entropy"] = _statistics(hidden.float() @ weight.float().t())
        state["g_hidden"], state["g_weight"] = torch.empty_like(hidden), torch.empty_like(weight)
    # a trainer's scratch memory: at most a gigabyte and a half
    state["work"] = torch.empty(_head_room(case), dtype=torch.uint8, device="cuda")
    return state


def _head_room(case):
    return (64 << 20) if case["op"] == "head" else (1536 << 20)


def prepare(case, seed):
    seed = int(seed) + 0x51A0000
    if case["op"] == "plan":
        return _prepare_plan(case, seed)
    return _prepare_scores(case, seed) if case["op"].startswith("scores") else _prepare_head(case, seed)


# ---- the plain forms -------------------------------------------------------------------------


def _plain_plan(s):
    page, tables = s["page"], s["tables"]
    cached, new, room = s["cached"], s["new"], len(s["ids"])
    n, width = tables.shape
    offsets = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(new, 0)
    held = (cached + page - 1) // page if s["held"] is None else s["held"]
    lengths = cached + new
    pages = torch.maximum(held, (lengths + page - 1) // page)
    before = torch.cumsum(pages - held, 0) - (pages - held)
    col = torch.arange(width, dtype=torch.int32, device="cuda")
    fresh = (col >= held[:, None]) & (col < pages[:, None])
    place = (s["count"] - 1) - (before[:, None] + (col - held[:, None]))
    tables = torch.where(fresh, s["free"][place.clamp(0, len(s["free"]) - 1)], tables)
    t = torch.arange(room, dtype=torch.int32, device="cuda")
    request = torch.searchsorted(offsets[1:], t, right=True)
    real = request < n
    r = request.clamp(max=n - 1)
    position = cached[r] + t - offsets[r]
    block = torch.div(position, page, rounding_mode="floor").clamp(0, width - 1)
    slot = tables[r, block].long() * page + position % page
    following = torch.cat([s["ids"][1:], s["ids"][:1]])
    target = torch.where(real & (t + 1 < offsets[r + 1]), following, -1)
    result = torch.stack([offsets[-1].long(), s["count"][0] - (pages - held).sum()])
    return dict(offsets=offsets, lengths=lengths, pages=pages, tables=tables, slots=torch.where(real, slot, -1),
                positions=torch.where(real, position, 0).int(), requests=torch.where(real, request, -1).int(),
                targets=target.int(), result=result)


def _plain_from(x, targets):
    """Log probabilities, statistics and entropy of rows of 32-bit logits."""
    m = x.amax(1, keepdim=True)
    d = x - m
    e = d.exp()
    s = e.sum(1, keepdim=True)
    entropy = s.log() - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / s
    given = d.gather(1, targets.clamp(min=0).long()[:, None]) - s.log()
    logprobs = torch.where(targets < 0, 0.0, given[:, 0])
    return dict(logprobs=logprobs, stats=torch.cat([m, s.log()], 1), entropy=entropy[:, 0])


def _plain_scores(s):
    x = s["logits"].float()
    out = _plain_from(x, s["targets"])
    if s["top"]:
        # order by value, the lowest index first among equals: one whole number for each entry
        bits = x.view(torch.int32) if x.is_contiguous() else x.contiguous().view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32
        key += (0x7FFFFFFF - torch.arange(x.shape[1], device="cuda"))
        best = torch.topk(key, s["top"], dim=1).values
        ids = 0x7FFFFFFF - (best & 0xFFFFFFFF)
        values = x.gather(1, ids)
        out["alt_ids"] = torch.where(values == -math.inf, -1, ids).int()
        out["alt_logprobs"] = values - out["stats"][:, :1] - out["stats"][:, 1:]
    return out


def _plain_logits_grad(x, s):
    lp = x - s["stats"][:, :1] - s["stats"][:, 1:]
    p = lp.exp()
    g = -p * s["g_logprobs"][:, None]
    g.masked_fill_((s["targets"] < 0)[:, None], 0.0)
    g -= s["g_entropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    rows = torch.arange(len(g), device="cuda")
    given = torch.where(s["targets"] < 0, 0.0, s["g_logprobs"])
    g[rows, s["targets"].clamp(min=0).long()] += given
    return g


def _plain(s):
    op = s["op"]
    if op == "plan":
        return _plain_plan(s)
    if op == "scores":
        return _plain_scores(s)
    if op == "scores_grad":
        return dict(g_logits=_plain_logits_grad(s["logits"].float(), s).to(s["logits"].dtype))
    hidden, weight = s["hidden"].float(), s["weight"].float()
    x = hidden @ weight.t()
    if op == "head":
        return _plain_from(x, s["targets"])
    g = _plain_logits_grad(x, s)
    return dict(g_hidden=(g @ weight).to(s["hidden"].dtype), g_weight=(g.t() @ hidden).to(s["hidden"].dtype))


# ---- the framework's operators ---------------------------------------------------------------


def _own(s):
    import paper_2607_29678_amd as tt

    op, stream = s["op"], torch.cuda.current_stream().cuda_stream
    if op == "plan":
        tt.step_plan(s["cached"], s["new"], s["tables"], s["free"], s["count"], s["page"], s["offsets"], s["lengths"],
                     s["pages"], s["slots"], s["positions"], s["requests"], s["result"], held=s["held"], ids=s["ids"],
                     targets=s["targets"], stream=stream)
        return {k: s[k] for k in ("offsets", "lengths", "pages", "tables", "slots", "positions", "requests", "targets", "result")}
    if op == "scores":
        alt = (s["alt_ids"], s["alt_logprobs"]) if s["top"] else (None, None)
        tt.token_scores(s["logits"], s["targets"], s["logprobs"], s["stats"], s["entropy"], *alt, workspace=s["work"],
                        stream=stream)
        out = {k: s[k] for k in ("logprobs", "stats", "entropy")}
        return dict(out, alt_ids=alt[0], alt_logprobs=alt[1]) if s["top"] else out
    if op == "scores_grad":
        tt.token_scores_grad(s["logits"], s["targets"], s["stats"], s["entropy"], s["g_logprobs"], s["g_entropy"],
                             s["g_logits"], stream=stream)
        return dict(g_logits=s["g_logits"])
    if op == "head":
        tt.head_scores(s["hidden"], s["weight"], s["targets"], s["logprobs"], s["stats"], s["entropy"],
                       workspace=s["work"], stream=stream)
        return {k: s[k] for k in ("logprobs", "stats", "entropy")}
    tt.head_scores_grad(s["hidden"], s["weight"], s["targets"], s["stats"], s["entropy"], s["g_logprobs"], s["g_entropy"],
                        s["g_hidden"], s["g_weight"], workspace=s["work"], stream=stream)
    return dict(g_hidden=s["g_hidden"], g_weight=s["g_weight"])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Inputs read once, outputs written once; the products of the head forward, recomputed and both ways back."""
    op = case["op"]
    if op == "plan":
        n, t = case["requests"], case["tokens"]
        entries = t / case["page"] + n
        return {"bytes": 12.0 * n + 24.0 * t + 8.0 * entries + 16.0 * n, "flops": 0}
    rows, vocab = case["rows"], case["vocab"]
    if op == "scores":
        return {"bytes": rows * (vocab * BYTES[case["type"]] + 20.0 + 8.0 * case["top"]), "flops": 6.0 * rows * vocab}
    if op == "scores_grad":
        return {"bytes": rows * (2.0 * vocab * BYTES[case["type"]] + 24.0), "flops": 7.0 * rows * vocab}
    width, one = case["width"], 2.0 * rows * case["width"] * vocab
    if op == "head":
        return {"bytes": 2.0 * width * (rows + vocab) + 20.0 * rows, "flops": one}
    return {"bytes": 4.0 * width * (rows + vocab) + 24.0 * rows, "flops": 3 * one}


# ---- the definitions, in 64 bits -------------------------------------------------------------


def _exact_softmax(z):
    lse = torch.logsumexp(z, dim=1)
    lp = z - lse[:, None]
    return lse, lp


def exact(case, seed):
    if case["op"] == "plan":
        return None  # whole numbers: equal or wrong
    s = prepare(case, seed)
    given = s["targets"].long()
    one_hot = lambda v: (torch.arange(v, device="cuda")[None, :] == given[:, None])  # noqa: E731  (-1: no column)
    if case["op"] in ("scores", "head"):
        z = s["logits"].double() if case["op"] == "scores" else torch.matmul(s["hidden"].double(), s["weight"].double().t())
        lse, lp = _exact_softmax(z)
        top = torch.max(z, dim=1).values
        out = dict(logprobs=torch.where(one_hot(z.shape[1]), lp, torch.zeros((), dtype=torch.float64, device="cuda")).sum(1),
                   stats=torch.stack([top, lse - top], dim=1), entropy=-torch.special.xlogy(lp.exp(), lp.exp()).sum(1))
        if case["op"] == "scores" and case["top"]:
            out["alt_ids"] = None
            out["alt_logprobs"] = torch.sort(lp, dim=1, descending=True).values[:, :case["top"]].contiguous()
        return out
    # the gradient of sum(a * logprob + b * entropy) over the rows
    z = s["logits"].double() if case["op"] == "scores_grad" else torch.matmul(s["hidden"].double(), s["weight"].double().t())
    a, b = s["g_logprobs"].double(), s["g_entropy"].double()
    _, lp = _exact_softmax(z)
    p = lp.exp()
    plogp = torch.special.xlogy(p, p)
    d = (one_hot(z.shape[1]).double() - p) * (a * (given >= 0))[:, None]
    d = d - b[:, None] * (plogp - p * plogp.sum(1, keepdim=True))
    if case["op"] == "scores_grad":
        return dict(g_logits=d)
    return dict(g_hidden=torch.matmul(d, s["weight"].double()), g_weight=torch.matmul(d.t().contiguous(), s["hidden"].double()))
