"""``tt_cache_attention`` where scores lie far apart or far from zero: what the exponents and the weights have to hold."""

import math
import types

import pytest

torch = pytest.importorskip("torch")
from paper_2607_29678_amd import cache_attention, cache_attention_workspace  # noqa: E402

pytestmark = pytest.mark.gpu
BF, H = torch.bfloat16, torch.float16


def step(requests, heads, k, v, page=16):
    """A step of (cached, new) tokens whose requests all hold the same tokens: k and v [tokens, kv, dim]."""
    n, kv, dim = k.shape
    held = -(-n // page)
    cache = [torch.zeros(held * page, kv, dim, dtype=k.dtype) for _ in range(2)]
    for c, x in zip(cache, (k, v)):
        c[:n] = x
    new = torch.tensor([0] + [f for _, f in requests]).cumsum(0).int()
    return types.SimpleNamespace(
        requests=requests, heads=heads, kv=kv, dim=dim, dtype=k.dtype, tokens=int(new[-1]), offsets=new.cuda(),
        keys=cache[0].view(held, page, kv, dim).cuda(), values=cache[1].view(held, page, kv, dim).cuda(),
        tables=torch.arange(held, dtype=torch.int32).repeat(len(requests), 1).cuda(),
        lengths=torch.tensor([c + f for c, f in requests], dtype=torch.int32).cuda())


def run(s, queries, scale):
    out = torch.empty(s.tokens, s.heads, s.dim, dtype=s.dtype, device="cuda")
    sums = torch.empty(s.tokens, s.heads, device="cuda")
    need = cache_attention_workspace(s.tokens, len(s.requests), s.heads, s.kv, s.dim)
    work = torch.full((max(need, 1),), 0xA5, dtype=torch.uint8, device="cuda")
    cache_attention(queries.cuda(), s.keys, s.values, s.tables, s.offsets, s.lengths, out, sums, scale, workspace=work,
                    stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return out.cpu(), sums.cpu()


def positions(s):
    return [c + i for c, f in s.requests for i in range(f)]


@pytest.mark.parametrize("dtype", [BF, H])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("requests", [[(300, 1), (77, 1), (0, 1)], [(130, 150), (0, 90), (255, 1)]])
@pytest.mark.parametrize("scale", [3e6, 1.7e9, 1e20])
def test_scores_far_from_zero(gpu, requests, dim, dtype, scale):
    """Scores of whole numbers times a large scale: each token's largest one leaves nothing to the others.  The whole
    numbers are products without rounding, and 3e6 and more apart after scaling, so that the largest one's weight is the
    sum of all, a power of two, and the result is its value, exactly.  The logarithm of the sums is its score, with seven
    roundings by 2^-24 of it (the scale, log2(e), their product, the score's, ln 2, the product with it, the sum) and as many
    of an offset of at most 5."""
    n, kv, heads = 301, 2, 4
    g = torch.Generator().manual_seed(dim)
    k, v = torch.zeros(n, kv, dim), torch.randn(n, kv, dim, generator=g).to(dtype)
    # (different for every token; in two parts that both types hold)
    level = torch.stack([torch.randperm(n, generator=g) for _ in range(kv)], 1) - 150.0
    k[:, :, 3], k[:, :, 7] = torch.div(level, 16, rounding_mode="floor"), level % 16
    q = torch.zeros(sum(f for _, f in requests), heads, dim)
    q[:, :, 3], q[:, :, 7] = 16.0, 1.0
    s = step(requests, heads, k.to(dtype), v)
    out, sums = run(s, q.to(dtype), scale)
    for t, p in enumerate(positions(s)):
        for h in range(heads):
            best = int(level[:p + 1, h // 2].argmax())
            assert torch.equal(out[t, h], v[best, h // 2]), (t, p, h)
            want = float(level[best, h // 2]) * scale
            assert abs(float(sums[t, h]) - want) <= 7 * 2.0 ** -24 * (abs(want) + 5)
