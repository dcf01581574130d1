"""The operators between a step's plan and the scores of its tokens, as performance cases.

``append``: keys and values of a step's tokens into the slots of a paged cache, with the position
rotation applied on the way (to the queries too).  ``attention``: the step's queries over that
cache through the page tables, with an optional sliding window and first tokens that stay visible.
``adjust`` and ``adjust_grad``: penalties for repeated tokens, biases and masks on stored logits, and
the gradient.  Vocabulary sizes are those of the stored merge tables (1,281, 8,449, 50,257 and
100,257 entries).
"""

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
VOCABS = (1_281, 8_449, 50_257, 100_257)
HEADS = ((32, 8), (16, 16), (20, 4), (28, 4), (64, 8), (12, 12), (8, 1))  # of queries, of keys
PAGES = (8, 16, 16, 24, 32, 64, 128)


def listed():
    return [
        # a decode step of a busy server: one token a request, launch latency counts
        dict(name="append decode 96", op="append", tokens=96, context=4_000, heads=32, kv=8, dim=128, rotated=128,
             interleaved=False, page=16, type="bf16"),
        # a prefill of documents far into long contexts; the first half of each head is rotated, in neighbouring pairs
        dict(name="append prefill 30001", op="append", tokens=30_001, context=300_000, heads=20, kv=4, dim=96, rotated=48,
             interleaved=True, page=24, type="f16"),
        # a few short requests: latency
        dict(name="attention decode 4", op="attention", requests=4, tokens=4, context=700, heads=16, kv=16, dim=64, page=16,
             window=0, sinks=0, type="f16"),
        # a decode step of a busy server
        dict(name="attention decode 96", op="attention", requests=96, tokens=96, context=4_000, heads=32, kv=8, dim=128,
             page=16, window=0, sinks=0, type="bf16"),
        # two requests over whole books: few rows, long lengths
        dict(name="attention decode long 2", op="attention", requests=2, tokens=2, context=120_001, heads=28, kv=4, dim=128,
             page=64, window=0, sinks=0, type="bf16"),
        # five guessed tokens a request are checked, with a sliding window and four first tokens
        dict(name="attention window 64", op="attention", requests=64, tokens=320, context=20_000, heads=64, kv=8, dim=64,
             page=32, window=4_096, sinks=4, type="bf16"),
        # decode and chunked prefill in one step
        dict(name="attention mixed 33", op="attention", requests=33, tokens=2_081, context=6_000, heads=20, kv=4, dim=96,
             page=24, window=0, sinks=0, type="f16"),
        # the prefill of two documents
        dict(name="attention prefill 14001", op="attention", requests=2, tokens=14_001, context=0, heads=32, kv=8, dim=128,
             page=16, window=0, sinks=0, type="bf16"),
        # a decode step with penalties and a few biases
        dict(name="adjust decode 32", op="adjust", rows=32, vocab=50_257, history=700, biases=20, allowed=1.0, padded=False,
             type="bf16"),
        # constrained answers of a large batch: masks of a grammar's states, long histories
        dict(name="adjust constrained 512", op="adjust", rows=512, vocab=100_257, history=2_000, biases=0, allowed=0.05,
             padded=True, type="f32"),
        # training on a small vocabulary, the gradient back through penalties and masks
        dict(name="adjust grad 65", op="adjust_grad", rows=65, vocab=8_449, history=300, biases=0, allowed=0.3, padded=False,
             type="f16"),
        # policy gradient on answers that were sampled with penalties and masks
        dict(name="adjust grad 1536", op="adjust_grad", rows=1_536, vocab=100_257, history=1_000, biases=0, allowed=0.5,
             padded=False, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "attention", "adjust", "adjust_grad"))
    heads, kv = rng.choice(HEADS)
    dim, page, kind = rng.choice((64, 80, 96, 128, 128)), rng.choice(PAGES), rng.choice(("bf16", "bf16", "f16"))
    if op == "append":
        most = 30_001 * (2 * 20 + 4 * 4) * 96 // ((2 * heads + 4 * kv) * dim)
        return dict(op=op, tokens=_log(rng, 1, most), context=_log(rng, 1, 1_000_000), heads=heads, kv=kv, dim=dim,
                    rotated=rng.choice((dim, dim, dim // 2)), interleaved=rng.random() < 0.4, page=page, type=kind)
    if op == "attention":
        step = rng.choice(("decode", "decode", "guess", "mixed", "prefill"))
        window, sinks = rng.choice(((0, 0), (0, 0), (_log(rng, 100, 8_000), 0), (_log(rng, 100, 8_000), rng.choice((1, 4, 4, 30)))))
        if step == "decode":
            requests, context = _log(rng, 1, 300), _log(rng, 20, 100_000)
            tokens = requests
        elif step == "guess":
            requests, context = _log(rng, 1, 100), _log(rng, 100, 30_000)
            tokens = requests * rng.randint(2, 9)
        elif step == "mixed":
            requests, context = _log(rng, 2, 40), _log(rng, 100, 6_000)
            tokens = _log(rng, 2 * requests, 2_000)
        else:
            requests, context = _log(rng, 1, 8), 0
            tokens = _log(rng, 50 * requests, min(10_000, int((4e11 / (heads * dim)) ** 0.5)))
        context = min(context, 350_000 * 8 // (requests * kv))
        return dict(op=op, requests=requests, tokens=tokens, context=context, heads=heads, kv=kv, dim=dim, page=page,
                    window=window, sinks=sinks, type=kind)
    vocab = rng.choice(VOCABS + (_log(rng, 1_000, 100_000),))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    rows = _log(rng, 1, min(6_000, (150_000_000 if op == "adjust_grad" else 100_000_000) // (vocab * BYTES[kind] // 2)))
    return dict(op=op, rows=rows, vocab=vocab, history=_log(rng, 1, 4_000),
                biases=rng.choice((0, 0, 1, 20, 100)) if op == "adjust" else 0, allowed=rng.choice((1.0, 1.0, 0.5, 0.01)),
                padded=rng.random() < 0.3, type=kind)


# ---- inputs ----------------------------------------------------------------------------------


def _room(tokens):
    """Entries of the per-token arrays: a step is padded to a multiple of 8, as for a captured graph."""
    return -(-tokens // 8) * 8


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _lengths(case):
    """(cached, new) tokens of the requests of a step; a seed gives them another order."""
    n, tokens = case["requests"], case["tokens"]
    rng = np.random.RandomState((n * 7_919 + tokens * 31 + case["context"]) % (1 << 32))
    new = np.full(n, tokens // n, dtype=np.int64)
    if tokens >= 10 * n:  # long and short prompts; the rest decode one token
        w = np.where(rng.rand(n) < 0.6, rng.lognormal(0.0, 0.7, n), 0.0)
        w[rng.randint(n)] += 1.0
        new = 1 + np.floor((tokens - n) * w / w.sum()).astype(np.int64)
    rest = tokens - int(new.sum())
    new += rest // n
    new[:rest % n] += 1
    cached = np.zeros(n, dtype=np.int64)
    if case["context"]:
        cached = np.clip(rng.lognormal(math.log(case["context"]) - 0.08, 0.4, n), 1, 2 * case["context"]).astype(np.int64)
    return cached, new


def _normal(gen, shape, kind, size=1.0):
    """Normal values, made piece by piece."""
    out = torch.empty(shape, dtype=kind, device="cuda")
    for part in out.view(-1).split(1 << 27):
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda").mul_(size))
    return out


def _prepare_append(case, seed):
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.RandomState(seed % (1 << 32))
    tokens, page, heads, kv, dim = (case[k] for k in ("tokens", "page", "heads", "kv", "dim"))
    kind, room = TYPES[case["type"]], _room(case["tokens"])
    # requests of one token, or of prompts; each begins anywhere in a page
    slots, positions, used = np.full(room, -1, dtype=np.int64), np.zeros(room, dtype=np.int32), 0
    each = 1 if tokens <= 256 else -(-tokens // 16)
    pages = rng.permutation(-(-tokens // each) * (each // page + 2) + 8)
    for a in range(0, tokens, each):
        m = min(each, tokens - a)
        first = rng.randint(case["context"], 2 * case["context"] + 1)
        at = first % page + np.arange(m)
        slots[a:a + m] = pages[used + at // page] * page + at % page
        positions[a:a + m] = first + np.arange(m)
        used += int(at[-1]) // page + 1
    qkv = _normal(gen, (room, (heads + 2 * kv) * dim), kind)  # one projection's output: the three parts are views
    q, k, v = (x.view(room, -1, dim) for x in qkv.split((heads * dim, kv * dim, kv * dim), 1))
    base = 10_000.0 if case["context"] < 50_000 else 5_000_000.0
    pairs = case["rotated"] // 2
    return dict(op="append", queries=q, keys=k, values=v, slots=_dev(slots), positions=_dev(positions),
                frequencies=_dev((base ** (-np.arange(pairs) / pairs)).astype(np.float32)), interleaved=case["interleaved"],
                key_cache=_normal(gen, (len(pages), page, kv, dim), kind), value_cache=_normal(gen, (len(pages), page, kv, dim), kind),
                turned=torch.zeros(room, heads, dim, dtype=kind, device="cuda"))


def _prepare_attention(case, seed):
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.RandomState(seed % (1 << 32))
    page, heads, kv, dim, kind = case["page"], case["heads"], case["kv"], case["dim"], TYPES[case["type"]]
    cached, new = _lengths(case)
    order = rng.permutation(len(cached))
    cached, new = cached[order], new[order]
    lengths = cached + new
    held = -(-lengths // page)
    width = int(held.max()) + 2
    pages = rng.permutation(int(held.sum()) + 20).astype(np.int32)
    tables = np.full((len(held), width), -1, dtype=np.int32)
    tables[np.arange(width)[None, :] < held[:, None]] = pages[:held.sum()]
    room = _room(case["tokens"])
    return dict(op="attention", page=page, window=case["window"], sinks=case["sinks"], tables=_dev(tables),
                offsets=_dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), lengths=_dev(lengths.astype(np.int32)),
                most_new=int(new.max()), longest=int(lengths.max()), queries=_normal(gen, (room, heads, dim), kind, 1.5),
                key_cache=_normal(gen, (len(pages), page, kv, dim), kind), value_cache=_normal(gen, (len(pages), page, kv, dim), kind),
                out=torch.zeros(room, heads, dim, dtype=kind, device="cuda"),
                logsums=torch.zeros(room, heads, dtype=torch.float32, device="cuda"),
                work=torch.empty(192 << 20, dtype=torch.uint8, device="cuda"))  # a server's scratch memory


def _prepare_adjust(case, seed):
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.RandomState(seed % (1 << 32))
    rows, vocab, kind = case["rows"], case["vocab"], TYPES[case["type"]]
    pitch = -(-vocab // 64) * 64 if case["padded"] else vocab
    logits = _normal(gen, (rows, pitch), kind, 2.5)[:, :vocab]
    # texts repeat some tokens often: IDs fall off like a power
    lengths = rng.randint(0, 2 * case["history"] + 1, rows)
    draw_ids = lambda n: np.minimum(vocab * rng.rand(n) ** 4, vocab - 1).astype(np.int32)  # noqa: E731
    state = dict(op=case["op"], vocab=vocab, logits=logits, history=_dev(draw_ids(int(lengths.sum()))),
                 history_offsets=_dev(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)),
                 repetition=_dev((1.0 + 0.3 * rng.rand(rows)).astype(np.float32)), presence=None, frequency=None,
                 bias_ids=None, bias_values=None, bias_offsets=None, masks=None, mask_rows=None)
    if case["op"] == "adjust":
        state.update(presence=_dev(rng.rand(rows).astype(np.float32)), frequency=_dev((0.2 * rng.rand(rows)).astype(np.float32)))
    if case["biases"]:
        k = case["biases"]
        ids = np.argsort(rng.rand(rows, 4 * k), 1)[:, :k] * (vocab // (4 * k)) + rng.randint(0, vocab // (4 * k), (rows, k))
        state.update(bias_ids=_dev(ids.reshape(-1).astype(np.int32)), bias_values=_dev(rng.randn(rows * k).astype(np.float32) * 5),
                     bias_offsets=_dev(np.arange(rows + 1, dtype=np.int64) * k))
    if case["allowed"] < 1:  # states of a grammar; answers that are in none go unmasked
        allowed = torch.rand(16, -(-vocab // 32), 32, generator=gen, device="cuda") < case["allowed"]
        words = (allowed.long() << torch.arange(32, device="cuda")).sum(2)
        state.update(masks=torch.where(words >= 1 << 31, words - (1 << 32), words).int(),
                     mask_rows=_dev(np.where(rng.rand(rows) < 0.2, -1, rng.randint(0, 16, rows)).astype(np.int32)))
    if case["op"] == "adjust":
        state["out"] = torch.empty_like(logits, memory_format=torch.contiguous_format)
    else:
        state["grad_out"] = _normal(gen, (rows, vocab), kind, 1.0 / math.sqrt(rows))
        state["grad_logits"] = torch.empty(rows, vocab, dtype=kind, device="cuda")
    return state


def prepare(case, seed):
    seed = int(seed) + 0x7E50000
    if case["op"] == "append":
        return _prepare_append(case, seed)
    return _prepare_attention(case, seed) if case["op"] == "attention" else _prepare_adjust(case, seed)


# ---- the plain forms -------------------------------------------------------------------------


def _plain_rotate(x, positions, frequencies, interleaved):
    pairs = len(frequencies)
    angle = positions.double()[:, None, None] * frequencies.double()  # (far positions: an angle's turns are many)
    cos, sin = angle.cos().float(), angle.sin().float()
    y = x.float()
    turn, rest = y[..., :2 * pairs], y[..., 2 * pairs:]
    if interleaved:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = turn[..., :pairs], turn[..., pairs:]
        turn = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turn, rest], -1).to(x.dtype)


def _plain_append(s):
    rotate = lambda x: _plain_rotate(x, s["positions"], s["frequencies"], s["interleaved"])  # noqa: E731
    real = (s["slots"] >= 0)[:, None, None]
    # rows without a slot write what the first row writes, to the same place
    slots = torch.where(s["slots"] >= 0, s["slots"], s["slots"][0])
    for cache, rows in ((s["key_cache"], rotate(s["keys"])), (s["value_cache"], s["values"])):
        cache.view(-1, *cache.shape[2:])[slots] = torch.where(real, rows, rows[:1])
    return dict(key_cache=s["key_cache"], value_cache=s["value_cache"],
                turned=torch.where(real, rotate(s["queries"]), s["turned"]))


def _plain_attention(s):
    room, heads, dim = s["queries"].shape
    kv, n, page, longest, most = s["key_cache"].shape[2], len(s["lengths"]), s["page"], s["longest"], s["most_new"]
    out = torch.zeros(room + 1, heads, dim, dtype=s["queries"].dtype, device="cuda")
    logsums = torch.zeros(room + 1, heads, dtype=torch.float32, device="cuda")
    keys, i = torch.arange(longest, device="cuda"), torch.arange(most, device="cuda")
    at_once = max(1, (1 << 29) // (most * longest * heads))  # requests whose scores are held at once
    for r in range(0, n, at_once):
        offsets, lengths = s["offsets"][r:r + at_once + 1].long(), s["lengths"][r:r + at_once].long()
        m, new = len(lengths), offsets[1:] - offsets[:-1]
        slots = s["tables"][r:r + m].long()[:, keys // page].clamp(min=0) * page + keys % page
        k = s["key_cache"].view(-1, kv, dim)[slots].float().permute(0, 2, 3, 1).contiguous()  # [m, kv, dim, keys]
        v = s["value_cache"].view(-1, kv, dim)[slots].float().permute(0, 2, 1, 3).contiguous()
        rows = torch.where(i < new[:, None], offsets[:-1, None] + i, room)
        q = s["queries"][rows.clamp(max=room - 1)].float().view(m, most, kv, heads // kv, dim)
        q = q.permute(0, 2, 3, 1, 4).reshape(m, kv, heads // kv * most, dim)
        x = (torch.matmul(q, k) * dim ** -0.5).view(m, kv, heads // kv, most, longest)
        position = ((lengths - new)[:, None] + i)[..., None]
        seen = keys <= position
        if s["window"]:
            seen &= (keys > position - s["window"]) | (keys < s["sinks"])
        x.masked_fill_(~seen[:, None, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        y = torch.matmul(p.view(m, kv, -1, longest), v).view(m, kv, heads // kv, most, dim) / total
        out[rows] = y.permute(0, 3, 1, 2, 4).reshape(m, most, heads, dim).to(out.dtype)
        logsums[rows] = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(m, most, heads)
        del x, p, y, k, v
    return dict(out=out[:room], logsums=logsums[:room])


def _row_of(offsets, n):
    """The row that each of n entries of a list belongs to."""
    return torch.searchsorted(offsets[1:], torch.arange(n, device="cuda"), right=True)


def _counts(s):
    rows, vocab = s["logits"].shape
    counts = torch.zeros(rows * vocab, dtype=torch.int32, device="cuda")
    at = _row_of(s["history_offsets"], len(s["history"])) * vocab + s["history"]
    return counts.index_add_(0, at, torch.ones_like(s["history"])).view(rows, vocab)


def _banned(s):
    bits = (s["masks"][:, :, None] >> torch.arange(32, dtype=torch.int32, device="cuda")) & 1
    allowed = bits.bool().flatten(1)[:, :s["vocab"]]
    return ~allowed[s["mask_rows"].clamp(min=0).long()] & (s["mask_rows"] >= 0)[:, None]


def _plain_adjust(s):
    x, counts = s["logits"].float(), _counts(s)
    r = s["repetition"][:, None]
    y = torch.where(counts > 0, torch.where(x > 0, x / r, x * r) - s["presence"][:, None] - s["frequency"][:, None] * counts, x)
    if s["bias_ids"] is not None:
        at = _row_of(s["bias_offsets"], len(s["bias_ids"])) * s["vocab"] + s["bias_ids"]
        y.view(-1).index_add_(0, at, s["bias_values"])  # (a row's biases are of different tokens)
    if s["masks"] is not None:
        y.masked_fill_(_banned(s), -math.inf)
    return dict(out=y.to(s["logits"].dtype))


def _plain_adjust_grad(s):
    g, r = s["grad_out"].float(), s["repetition"][:, None]
    g = torch.where(_counts(s) > 0, torch.where(s["logits"] > 0, g / r, g * r), g)
    if s["masks"] is not None:
        g.masked_fill_(_banned(s), 0.0)
    return dict(grad_logits=g.to(s["logits"].dtype))


PLAIN = {"append": _plain_append, "attention": _plain_attention, "adjust": _plain_adjust, "adjust_grad": _plain_adjust_grad}


# ---- the framework's operators ---------------------------------------------------------------


def _own(s):
    import paper_2607_29678_amd as tt

    op, stream = s["op"], torch.cuda.current_stream().cuda_stream
    if op == "append":
        tt.cache_append(s["keys"], s["values"], s["key_cache"], s["value_cache"], s["slots"], positions=s["positions"],
                        frequencies=s["frequencies"], interleaved=s["interleaved"], queries=s["queries"], rotated=s["turned"],
                        stream=stream)
        return {k: s[k] for k in ("key_cache", "value_cache", "turned")}
    if op == "attention":
        tt.cache_attention(s["queries"], s["key_cache"], s["value_cache"], s["tables"], s["offsets"], s["lengths"], s["out"],
                           logsums=s["logsums"], window=s["window"], sinks=s["sinks"], workspace=s["work"], stream=stream)
        return {k: s[k] for k in ("out", "logsums")}
    if op == "adjust":
        tt.adjust_logits(s["logits"], s["out"], history=s["history"], history_offsets=s["history_offsets"],
                         repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"], bias_ids=s["bias_ids"],
                         bias_values=s["bias_values"], bias_offsets=s["bias_offsets"], masks=s["masks"],
                         mask_rows=s["mask_rows"], stream=stream)
        return dict(out=s["out"])
    tt.adjust_logits_grad(s["logits"], s["grad_out"], s["grad_logits"], history=s["history"],
                          history_offsets=s["history_offsets"], repetition=s["repetition"], masks=s["masks"],
                          mask_rows=s["mask_rows"], stream=stream)
    return dict(grad_logits=s["grad_logits"])


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


def _seen(case):
    """(key vectors of a head that a step has to read, pairs of a query and a key)."""
    cached, new = _lengths(case)
    window, sinks = case["window"] or 1 << 40, case["sinks"]
    first = np.maximum(0, cached + 1 - window)  # the first token in the window of a request's first query
    keys = cached + new - first + np.minimum(sinks, first)
    p = np.concatenate([c + np.arange(k) for c, k in zip(cached, new)]) + 1
    return int(keys.sum()), int((np.minimum(p, window) + np.minimum(sinks, np.maximum(0, p - window))).sum())


def work(case):
    """Inputs read once, outputs written once; two products of a query, a key and a value for each visible pair."""
    op = case["op"]
    one = BYTES[case["type"]]
    if op == "append":
        tokens, width = case["tokens"], (2 * case["heads"] + 4 * case["kv"]) * case["dim"]
        return {"bytes": tokens * (width * one + 12.0) + 2.0 * case["rotated"],
                "flops": 3.0 * tokens * (case["heads"] + case["kv"]) * case["rotated"]}
    if op == "attention":
        keys, pairs = _seen(case)
        rows, dim = case["tokens"] * case["heads"], case["dim"]
        return {"bytes": 2.0 * keys * case["kv"] * dim * one + 2.0 * rows * dim * one + 4.0 * rows + 4.0 * keys / case["page"],
                "flops": 4.0 * pairs * case["heads"] * dim}
    rows, vocab = case["rows"], case["vocab"]
    masks = vocab / 8.0 * min(16, rows) if case["allowed"] < 1 else 0.0
    own_bytes = 2.0 * vocab * one + 4.0 * case["history"] + 8.0 * case["biases"] + 24.0
    return {"bytes": rows * own_bytes + masks, "flops": 2.0 * rows * vocab}


# ---- the definitions, in 64 bits -------------------------------------------------------------


def _exact_append(s):
    slots, n = s["slots"], int((s["slots"] >= 0).sum())
    t = s["frequencies"].double() * s["positions"][:n].double()[:, None]
    spin = torch.polar(torch.ones_like(t), t)[:, None, :]

    def turn(x):
        x, m = x[:n].double(), 2 * t.shape[1]
        pairs = x[..., :m].unflatten(-1, (-1, 2)) if s["interleaved"] else x[..., :m].unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * spin)
        return torch.cat([z.flatten(-2) if s["interleaved"] else z.transpose(-1, -2).flatten(-2), x[..., m:]], -1)

    out = {k: s[k].double() for k in ("key_cache", "value_cache", "turned")}
    out["key_cache"].flatten(0, 1)[slots[:n]] = turn(s["keys"])
    out["value_cache"].flatten(0, 1)[slots[:n]] = s["values"][:n].double()
    out["turned"][:n] = turn(s["queries"])
    return out


def _exact_attention(s):
    room, heads, dim = s["queries"].shape
    out = torch.zeros(room, heads, dim, dtype=torch.float64, device="cuda")
    logsums = torch.zeros(room, heads, dtype=torch.float64, device="cuda")
    offsets, page, kv = s["offsets"].tolist(), s["page"], s["key_cache"].shape[2]
    for r, length in enumerate(s["lengths"].tolist()):
        a, b = offsets[r], offsets[r + 1]
        pages = s["tables"][r, :-(-length // page)].long()
        k, v = (s[c][pages].flatten(0, 1)[:length].double() for c in ("key_cache", "value_cache"))
        for t in range(a, b, 1_024):  # queries of a piece see the keys up to its last one
            e = min(b, t + 1_024)
            at = torch.arange(length - b + t, length - b + e, device="cuda")[:, None]
            j = torch.arange(length - b + e, device="cuda")
            hidden = j > at
            if s["window"]:
                hidden |= (j <= at - s["window"]) & (j >= s["sinks"])
            for h in range(heads):
                g = h // (heads // kv)
                z = torch.matmul(s["queries"][t:e, h].double(), k[:len(j), g].t().contiguous()) / math.sqrt(dim)
                z[hidden] = -math.inf
                logsums[t:e, h] = torch.logsumexp(z, 1)
                out[t:e, h] = torch.matmul(torch.softmax(z, 1), v[:len(j), g].contiguous())
    return dict(out=out, logsums=logsums)


def _exact_adjust(s):
    rows, vocab = s["logits"].shape
    x, offsets = s["logits"].double(), s["history_offsets"].tolist()
    gradient = s["op"] == "adjust_grad"
    y = s["grad_out"].double() if gradient else x.clone()
    rep = s["repetition"].double()
    for i in range(rows):
        ids, times = torch.unique(s["history"][offsets[i]:offsets[i + 1]].long(), return_counts=True)
        factor = torch.where(x[i, ids] > 0, 1 / rep[i], rep[i])
        y[i, ids] *= factor
        if not gradient:
            y[i, ids] -= s["presence"][i].double() + s["frequency"][i].double() * times
        if s["bias_ids"] is not None:
            k = len(s["bias_ids"]) // rows
            y[i, s["bias_ids"][i * k:(i + 1) * k].long()] += s["bias_values"][i * k:(i + 1) * k].double()
        if s["masks"] is not None and int(s["mask_rows"][i]) >= 0:
            words = s["masks"][int(s["mask_rows"][i])].long() & 0xFFFFFFFF
            j = torch.arange(vocab, device="cuda")
            y[i, (words[j // 32] // 2 ** (j % 32)) % 2 == 0] = 0.0 if gradient else -math.inf
    return {"grad_logits" if gradient else "out": y}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention}.get(case["op"], _exact_adjust)(s)
