"""Plain 64-bit forms of the calls on a paged cache and on stored logits, their tolerances, and caches to run them on."""

import math

import torch

U32 = 2.0 ** -24
UNIT = {torch.float32: U32, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half a step, relative
SMALL = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}  # half the smallest step


def rotate(x, positions, frequencies, interleaved):
    """float64 [tokens, heads, dim] rotated, and the size of the terms of each result."""
    pairs = 0 if frequencies is None else len(frequencies)
    y, size = x.clone(), x.abs()
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, pairs + i)
        angle = (positions.double() * frequencies[i].double())[:, None]
        y[..., a] = x[..., a] * angle.cos() - x[..., b] * angle.sin()
        y[..., b] = x[..., a] * angle.sin() + x[..., b] * angle.cos()
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def rotate_tolerance(want, size, dtype):
    """An angle in half turns is at most 1, rounded to 32 bits (pi * 2^-24), its cosine and sine are good to 2 units of
    theirs (2 * 2^-23), two products and a sum round by 2^-24 each, and the result is rounded to its type.  64-bit angles
    differ by position * frequency * 2^-52, some 10^-10 at 10^6."""
    off = size * (math.pi + 4 + 3) * U32 + size * 1e-9
    return off + UNIT[dtype] * (want.abs() + off) + SMALL[dtype]


LAYOUTS = {"slots": (0, 1, 2), "heads": (0, 2, 1), "apart": (2, 0, 1)}  # order of pages, slots, heads in memory


def empty_cache(pages, page, kv, dim, dtype, layout="slots", fill=math.nan, device="cuda"):
    """[pages, page, kv, dim] whose first three dimensions lie in memory in this order."""
    order = LAYOUTS[layout]
    size = (pages, page, kv)
    t = torch.full([size[i] for i in order] + [dim], fill, dtype=dtype, device=device)
    back = [order.index(i) for i in range(3)] + [3]
    return t.permute(back)


class Step:
    """Queries, a cache and tables for requests of (cached, new) tokens; slots that no request holds are NaN."""

    def __init__(self, requests, heads, kv, dim, page, dtype, layout="slots", seed=0, room=None, q_size=1.0, extra=3):
        g = torch.Generator().manual_seed(seed)
        self.requests, self.heads, self.kv, self.dim, self.page, self.dtype = requests, heads, kv, dim, page, dtype
        lengths = [c + f for c, f in requests]
        held = [-(-n // page) for n in lengths]
        n_pages = sum(held) + extra
        numbers = torch.randperm(n_pages, generator=g)
        self.width = max([1] + held) + 1
        tables = torch.full((len(requests), self.width), -1, dtype=torch.int32)
        self.k, self.v, used = [], [], 0
        keys, values = (empty_cache(n_pages, page, kv, dim, dtype, layout, device="cpu") for _ in range(2))
        for r, n in enumerate(lengths):
            k, v = (torch.randn(n, kv, dim, generator=g).to(dtype) for _ in range(2))
            mine = numbers[used:used + held[r]]
            used += held[r]
            tables[r, :held[r]] = mine.int()
            for i in range(held[r]):
                m = min(page, n - i * page)
                keys[mine[i], :m] = k[i * page:i * page + m]
                values[mine[i], :m] = v[i * page:i * page + m]
            self.k.append(k)
            self.v.append(v)
        self.tables = tables.cuda()
        self.key_cache, self.value_cache = (self._to_device(x) for x in (keys, values))
        self.offsets = torch.tensor([0] + [f for _, f in requests]).cumsum(0).int().cuda()
        self.lengths = torch.tensor(lengths, dtype=torch.int32).cuda()
        self.tokens = sum(f for _, f in requests)
        self.room = self.tokens if room is None else room
        self.q = (torch.randn(self.room, heads, dim, generator=g) * q_size).to(dtype)
        self.queries = self.q.cuda()

    @staticmethod
    def _to_device(t):
        out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
        return out.copy_(t)

    def reference(self, window=0, sinks=0, scale=None, rows=None):
        """(out, logsums, tolerances of both) in float64 for the step's tokens (rows: only these)."""
        scale = self.dim ** -0.5 if scale is None else scale
        u, group = UNIT[self.dtype], self.heads // self.kv
        out = torch.zeros(self.tokens, self.heads, self.dim, dtype=torch.float64)
        sums = torch.full((self.tokens, self.heads), -math.inf, dtype=torch.float64)
        tol, sums_tol = torch.zeros_like(out), torch.zeros_like(sums)
        t = 0
        for (cached, new), k, v in zip(self.requests, self.k, self.v):
            j = torch.arange(cached + new)
            k, v = k.double().cuda(), v.double().cuda()
            for i in range(new):
                if rows is None or t in rows:
                    p = cached + i
                    seen = (j <= p) & ((j > p - window) | (j < sinks)) if window else j <= p
                    q = self.q[t].double().cuda().view(self.kv, group, self.dim)
                    ks, vs = (x[seen.cuda()].permute(1, 0, 2).contiguous() for x in (k, v))
                    x = (q[:, :, None] * ks[:, None]).sum(3) * scale  # [kv, group, keys]
                    terms = (q.abs()[:, :, None] * ks.abs()[:, None]).sum(3).amax(2) * scale
                    n = ks.shape[1]
                    top = x.amax(2, keepdim=True)
                    e = (x - top).exp()
                    total = e.sum(2, keepdim=True)
                    w = e / total
                    y = torch.matmul(w, vs)
                    size = torch.matmul(w, vs.abs())
                    # a score: sums of dim products and three roundings of the exponent, each at most `deep` large; an
                    # exponential 2 units, sums of n terms; the weights are rounded to the type once, and so is the result.
                    # A weight below the type's normal range (f16) is off by half its smallest step, relative to a
                    # largest of at least 1.
                    deep = (top - x.amin(2, keepdim=True))[..., 0].clamp(max=90)
                    e_x = U32 * ((self.dim + 4) * terms + 4 * (deep + top[..., 0].abs()))
                    rel = (2 * e_x + U32 * (n + 16))[..., None]
                    off = size * (u + rel) + n * SMALL[self.dtype] * vs.abs().amax() / total
                    full = off + u * (y.abs() + off) + SMALL[self.dtype]
                    ls = (top + total.log())[..., 0]
                    out[t], tol[t] = y.reshape(self.heads, -1).cpu(), full.reshape(self.heads, -1).cpu()
                    sums[t] = ls.reshape(-1).cpu()
                    sums_tol[t] = (e_x + U32 * (n + 16 + 4 * ls.abs())).reshape(-1).cpu()
                t += 1
        return out, sums, tol, sums_tol


def adjusted(x, history, repetition, presence, frequency, biases, allowed, grad=None):
    """float64 rows adjusted (or the gradient ``grad`` passed back), and the size of their terms.

    history, biases: a list a row, of IDs and of (ID, value) pairs; allowed: a bool row or None a row, or "bad"."""
    y = (x if grad is None else grad).clone()
    size = y.abs()
    rows, vocab = x.shape
    for r in range(rows):
        counts = {}
        for j in history[r] if history else ():
            if 0 <= j < vocab:
                counts[j] = counts.get(j, 0) + 1
        for j, n in counts.items():
            rho = 1.0 if repetition is None else float(repetition[r])
            y[r, j] = y[r, j] / rho if x[r, j] > 0 else y[r, j] * rho
            size[r, j] = y[r, j].abs()
            if grad is None:
                a = 0.0 if presence is None else float(presence[r])
                b = 0.0 if frequency is None else float(frequency[r])
                y[r, j] -= a + b * n
                size[r, j] += abs(a) + abs(b) * n
        for j, value in dict(biases[r] if biases and grad is None else ()).items():
            if 0 <= j < vocab:
                y[r, j] += value
                size[r, j] += abs(value)
        if allowed and isinstance(allowed[r], str):
            y[r] = math.nan
        elif allowed and allowed[r] is not None:
            y[r, ~allowed[r]] = -math.inf if grad is None else 0.0
    return y, size


def adjusted_tolerance(want, size, dtype):
    """At most five operations in 32 bits, none of more than the terms' size, and one rounding to the type."""
    off = 5 * U32 * size
    return off + UNIT[dtype] * (want.abs() + off) + SMALL[dtype]
