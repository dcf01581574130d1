"""``tt_cache_append`` against a plain 64-bit rotation: layouts, strides, orders, positions, tokens without a slot."""

import math

import pytest

torch = pytest.importorskip("torch")
from cache_reference import LAYOUTS, empty_cache, rotate, rotate_tolerance  # noqa: E402
from model_reference import close  # noqa: E402
from paper_2607_29678_amd import cache_append  # noqa: E402

pytestmark = pytest.mark.gpu
BF, H = torch.bfloat16, torch.float16


def freqs(pairs, base=10_000.0):
    return (base ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))).float().cuda()


def check(tokens, heads, kv, dim, pairs, interleaved, page, dtype, layout="slots", seed=0, far=5_000, skip=(), gap=0, lead=0,
          in_place=False, queries=True):
    g = torch.Generator().manual_seed(seed)
    width = (heads + 2 * kv) * dim + gap
    flat = torch.randn(tokens * width + lead, generator=g).to(dtype).cuda()[lead:].view(tokens, width)
    q, k, v = (flat[:, a * dim:b * dim].unflatten(1, (b - a, dim)) for a, b in
               ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    pages = tokens // page + 5
    keys, values = (empty_cache(pages, page, kv, dim, dtype, layout, fill=7.0) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g)[:tokens]
    for i, bad in enumerate(skip):
        slots[(i * 7) % tokens] = bad if bad < 0 else pages * page + bad
    positions = torch.randint(0, far, (tokens,), generator=g).int()
    positions[0] = far - 1
    f = freqs(pairs) if pairs else None
    source = q.clone()
    turned = (q if in_place else torch.full_like(source, 9.0)) if queries else None
    cache_append(k, v, keys, values, slots.cuda(), positions.cuda() if pairs else None, f, interleaved,
                 q if queries else None, turned, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    real = [t for t in range(tokens) if 0 <= slots[t] < pages * page]
    got_k, got_v = keys.reshape(-1, kv, dim).cpu(), values.reshape(-1, kv, dim).cpu()
    want, size = rotate(k.double().cpu()[real], positions[real], None if f is None else f.cpu(), interleaved)
    close(got_k[slots[real]], want, rotate_tolerance(want, size, dtype))
    assert torch.equal(got_k[slots[real]][..., 2 * pairs:], k.cpu()[real][..., 2 * pairs:])
    assert torch.equal(got_v[slots[real]], v.cpu()[real])
    others = torch.ones(pages * page, dtype=torch.bool)
    others[slots[real]] = False
    assert bool((got_k[others] == 7).all()) and bool((got_v[others] == 7).all())
    if queries:
        want, size = rotate(source.double().cpu()[real], positions[real], None if f is None else f.cpu(), interleaved)
        close(turned.cpu()[real], want, rotate_tolerance(want, size, dtype))
        rest = [t for t in range(tokens) if t not in set(real)]
        assert torch.equal(turned.cpu()[rest], (source if in_place else torch.full_like(source, 9.0)).cpu()[rest])


@pytest.mark.parametrize("dtype", [BF, H])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv,dim,pairs", [(32, 8, 128, 64), (20, 4, 96, 24), (4, 4, 64, 32), (3, 1, 80, 40), (5, 5, 8, 4),
                                                (2, 1, 256, 128), (6, 2, 40, 5), (7, 1, 24, 3), (4, 2, 64, 1), (8, 2, 128, 4)])
def test_heads(gpu, heads, kv, dim, pairs, interleaved, dtype):
    check(37, heads, kv, dim, pairs, interleaved, 16, dtype)


@pytest.mark.parametrize("tokens", [1, 2, 7, 255, 1_024, 3_001, 9_001])
def test_tokens(gpu, tokens):
    check(tokens, 4, 2, 64, 32, False, 16, BF, seed=tokens)
    check(tokens, 4, 2, 64, 16, True, 24, H, seed=tokens)


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("page", [1, 3, 16, 128])
def test_cache_layouts(gpu, layout, page):
    check(50, 4, 2, 64, 32, False, page, BF, layout)


@pytest.mark.parametrize("far", [1_000_000, 2**31 - 1])
def test_far_positions(gpu, far):
    check(64, 4, 2, 128, 64, False, 16, H, far=far)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("lead,gap", [(1, 0), (0, 3), (8, 8), (4, 4)])
def test_rows_off_their_alignment(gpu, lead, gap, interleaved):
    check(33, 6, 2, 64, 32, interleaved, 16, BF, lead=lead, gap=gap)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pairs,interleaved", [(32, False), (32, True), (5, False), (5, True), (0, False)])
def test_tokens_without_a_slot(gpu, in_place, pairs, interleaved):
    check(40, 4, 2, 64, pairs, interleaved, 16, BF, skip=(-1, -1, -5, 0, 10**9, -2**40), in_place=in_place)


def test_no_queries(gpu):
    check(40, 4, 2, 64, 32, False, 16, BF, queries=False)
    check(40, 4, 2, 64, 0, False, 16, H, queries=False)


def test_nothing(gpu):
    z = lambda *s: torch.zeros(s, dtype=BF, device="cuda")  # noqa: E731
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    keys = z(2, 16, 2, 64)
    cache_append(z(0, 2, 64), z(0, 2, 64), keys, z(2, 16, 2, 64), none)
    # a cache without pages takes nothing
    cache_append(z(3, 2, 64) + 1, z(3, 2, 64), z(0, 16, 2, 64), z(0, 16, 2, 64), torch.arange(3, device="cuda"))
    torch.cuda.synchronize()
    assert bool((keys == 0).all())


def test_special_values_stay_in_their_pair(gpu):
    k = torch.ones(2, 1, 64, dtype=BF, device="cuda")
    k[0, 0, 3], k[1, 0, 40] = math.nan, math.inf
    keys, values = (empty_cache(1, 4, 1, 64, BF, fill=0.0) for _ in range(2))
    cache_append(k, k, keys, values, torch.tensor([2, 0], device="cuda"), torch.tensor([5, 9], dtype=torch.int32, device="cuda"),
                 freqs(32))
    got = keys.reshape(4, 64).float().cpu()
    assert torch.nonzero(~torch.isfinite(got)).tolist() == [[0, 8], [0, 40], [2, 3], [2, 35]]


def test_slots_past_32_bits(gpu):
    # elements behind the 2^31st, in a cache of 2 x 4.5 GB
    pages, page, kv, dim = 70_000, 16, 16, 128
    keys, values = (torch.zeros(pages, page, kv, dim, dtype=BF, device="cuda") for _ in range(2))
    slots = torch.tensor([pages * page - 1, 3, 2**31 // (kv * dim), 2**31 // (kv * dim) + 1], device="cuda")
    k, v = (torch.randn(4, kv, dim, device="cuda").to(BF) for _ in range(2))
    cache_append(k, v, keys, values, slots)
    assert torch.equal(keys.view(-1, kv, dim)[slots], k) and torch.equal(values.view(-1, kv, dim)[slots], v)
    assert int((keys.view(-1, kv * dim) != 0).any(1).sum()) == 4
