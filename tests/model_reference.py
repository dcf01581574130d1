"""Plain 64-bit forms of the operators of ``toktier_model.h``, and the errors that their 32-bit sums may have."""

import math

import numpy as np
import torch

INF = math.inf


def plan(cached, fresh, held, page_size, tables, free, count, ids, room):
    """The step plan by loops over requests and tokens; tables are changed in place.  Returns a dict of lists."""
    n, width = tables.shape
    out = dict(offsets=[0], lengths=[], pages=[], slots=[-1] * room, positions=[0] * room, requests=[-1] * room,
               targets=[-1] * room)
    had = [(-(-int(c) // page_size) if held is None else int(h)) for c, h in zip(cached, cached if held is None else held)]
    bad = not 0 <= count <= len(free)
    take = []
    for r in range(n):
        c, f = int(cached[r]), int(fresh[r])
        need = -(-(c + f) // page_size)
        bad |= c < 0 or f < 0 or had[r] < 0 or c + f > 2**31 - 1 or need > width or had[r] > width
        take.append(max(0, need - had[r]))
    total = sum(max(0, int(f)) for f in fresh)
    bad |= total > room
    short = sum(take) > count
    if bad or short:
        out.update(offsets=[0] * (n + 1), lengths=[0] * n, pages=[max(0, h) for h in had], result=[-9 if bad else -8, count])
        return out
    t = 0
    for r in range(n):
        for j in range(take[r]):
            count -= 1
            tables[r, had[r] + j] = free[count]
        for i in range(int(fresh[r])):
            pos = int(cached[r]) + i
            out["positions"][t], out["requests"][t] = pos, r
            out["slots"][t] = int(tables[r, pos // page_size]) * page_size + pos % page_size
            out["targets"][t] = int(ids[t + 1]) if i + 1 < int(fresh[r]) else -1
            t += 1
        out["offsets"].append(t)
        out["lengths"].append(int(cached[r]) + int(fresh[r]))
        out["pages"].append(had[r] + take[r])
    out["result"] = [t, count]
    return out


def scores(z, targets, scale=1.0, n_alt=0):
    """Log probabilities, statistics, entropy and alternatives of float64 logits z [rows, vocab]."""
    rows, vocab = z.shape
    x = z * scale
    bad = torch.isnan(z).any(1) | (z == INF).any(1)
    none = (z == -INF).all(1) & ~bad
    fine = ~(bad | none)
    top = z.amax(1)
    safe = torch.where(fine[:, None], x - (top * scale)[:, None], torch.zeros_like(x))  # (masks may be huge)
    log_s = torch.logsumexp(safe, 1)
    lp = safe - log_s[:, None]
    lp = torch.where(fine[:, None], lp, torch.full_like(lp, -INF))
    lp[bad] = math.nan
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    entropy = torch.where(bad, torch.full_like(entropy, math.nan), entropy)
    stats = torch.stack([top, log_s], 1)
    stats[none] = -INF
    stats[bad] = math.nan
    t = targets.long()
    given = lp.gather(1, t.clamp(0, vocab - 1)[:, None])[:, 0]
    given = torch.where(t < 0, torch.zeros_like(given), torch.where(t >= vocab, torch.full_like(given, math.nan), given))
    out = dict(logprobs=given, stats=stats, entropy=entropy, lp=lp, p=p)
    if n_alt:
        ids = torch.full((rows, n_alt), -1, dtype=torch.int64)
        alt = torch.full((rows, n_alt), -INF, dtype=torch.float64)
        zc, lc = z.cpu().numpy(), lp.cpu()
        for r in range(rows):
            if bad[r]:
                alt[r] = math.nan
                continue
            order = np.lexsort((np.arange(vocab), -(zc[r] + 0.0)))[:n_alt]  # by value, then by index
            order = [int(i) for i in order if zc[r, i] > -INF]
            ids[r, :len(order)] = torch.tensor(order, dtype=torch.int64)
            alt[r, :len(order)] = lc[r, order]
        out.update(alt_ids=ids, alt_logprobs=alt)
    return out


def logits_grad(z, targets, g_lp, g_e, scale=1.0):
    """Gradient of sum(g_lp * logprob + g_e * entropy) with respect to z, and the sum of the sizes of its terms."""
    s = scores(z, targets, scale)
    p, h = s["p"], s["entropy"]
    gl = torch.where(targets < 0, torch.zeros_like(g_lp), g_lp)
    hit = torch.zeros_like(z)
    keep = (targets >= 0) & (targets < z.shape[1])
    hit[keep, targets[keep].long()] = 1.0
    plogp = torch.where(p > 0, p * torch.where(p > 0, s["lp"], torch.zeros_like(p)), torch.zeros_like(p))
    g = scale * (gl[:, None] * (hit - p) - g_e[:, None] * (plogp + p * h[:, None]))
    size = scale * (gl.abs()[:, None] * (hit + p) + g_e.abs()[:, None] * (plogp.abs() + p * h[:, None]))
    empty = (z == -INF).all(1) | ((gl == 0) & (g_e == 0))
    g[empty], size[empty] = 0.0, 0.0
    return g, size


U32 = 2.0 ** -24  # half a unit in the last place of a 32-bit float


def depth_of(lp):
    """[rows] how far below 0 the deepest log probability lies whose probability is not 0 in 32 bits."""
    seen = torch.isfinite(lp) & (lp > -104)
    return torch.where(seen, -lp, torch.zeros_like(lp)).amax(1)


def score_error(vocab, deepest, logit_error=0.0):
    """Bound of a log probability's error: the exponents (at most ``deepest`` below the largest, three roundings of
    them), the exponential and the logarithm (2 units each), a thread's sum of vocab / 256 terms and the tree above
    it, and twice the error of the logits themselves."""
    return U32 * (4 * deepest + 16 + vocab / 256 + 32) + 2 * logit_error


# unit roundoff (24, 8 and 11 bits of precision) and half the smallest step
ROUNDING = {torch.float32: (U32, 0.0), torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def close(got, want, tol):
    """got (any type) equals want (float64) up to tol, with equal infinities and NaNs; tol broadcasts."""
    got, want = got.double().cpu(), want.cpu()
    tol = torch.as_tensor(tol, dtype=torch.float64).cpu()
    special = ~torch.isfinite(want)
    same = torch.where(torch.isnan(want), torch.isnan(got), got == want)
    off = (got - want).abs()
    ok = torch.where(special, same, off <= tol)
    if not bool(ok.all()):
        i = torch.nonzero(~ok)[0].tolist()
        raise AssertionError("%d of %d values are off, the first at %s: %r, not %r (tolerance %r)"
                             % (int((~ok).sum()), ok.numel(), i, float(got[tuple(i)]), float(want[tuple(i)]),
                                float(tol.expand_as(got)[tuple(i)])))
