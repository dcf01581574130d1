"""The step plan against loops over requests and tokens: every value is a whole number."""

import numpy as np
import pytest

import model_reference as ref

pytestmark = pytest.mark.gpu


def make(rng, n, page, kind, room_over=5, held_over=0, zeros=0.2, most_cached=300, most_fresh=40):
    cached = rng.integers(0, most_cached + 1, n)
    fresh = np.ones(n, dtype=np.int64) if kind == "decode" else rng.integers(0, most_fresh + 1, n)
    fresh = np.where(rng.random(n) < zeros, 0, fresh)
    cached = np.where(rng.random(n) < zeros, 0, cached)
    # some lengths end exactly with a page
    cached = np.where(rng.random(n) < 0.2, cached // page * page, cached)
    held = -(-cached // page)
    if held_over:
        held = held + rng.integers(0, held_over + 1, n)
    need = np.maximum(held, -(-(cached + fresh) // page))
    width = int(need.max(initial=0)) + 1
    take = int((need - held).sum())
    pages = rng.permutation(2**20)[: int(held.sum()) + take + 7].astype(np.int32)
    tables = np.full((n, width), -7, dtype=np.int32)
    at = 0
    for r in range(n):
        tables[r, : held[r]] = pages[at: at + held[r]]
        at += held[r]
    free = pages[at:]
    room = int(fresh.sum()) + room_over
    ids = rng.integers(0, 2**31 - 1, room).astype(np.int32)
    return dict(cached=cached.astype(np.int32), fresh=fresh.astype(np.int32), held=held.astype(np.int32) if held_over else None,
                tables=tables, free=free, count=len(free), page=page, ids=ids, room=room)


def run(torch, c, stream=None, use_ids=True, stride_over=0):
    from paper_2607_29678_amd import step_plan

    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda")  # noqa: E731
    n, room = len(c["cached"]), c["room"]
    i32 = lambda k: torch.full((k,), -99, dtype=torch.int32, device="cuda")  # noqa: E731
    wide = torch.full((n, c["tables"].shape[1] + stride_over), -55, dtype=torch.int32, device="cuda")
    tables = wide[:, : c["tables"].shape[1]]
    tables.copy_(dev(c["tables"]))
    o = dict(offsets=i32(n + 1), lengths=i32(n), pages=i32(n), positions=i32(room), requests=i32(room),
             slots=torch.full((room,), -99, dtype=torch.int64, device="cuda"),
             result=torch.full((2,), -99, dtype=torch.int64, device="cuda"))
    targets = i32(room) if use_ids else None
    step_plan(dev(c["cached"]), dev(c["fresh"]), tables, dev(c["free"]),
              torch.tensor([c["count"]], dtype=torch.int64, device="cuda"), c["page"], o["offsets"], o["lengths"], o["pages"],
              o["slots"], o["positions"], o["requests"], o["result"], held=dev(c["held"]),
              ids=dev(c["ids"]) if use_ids else None, targets=targets, stream=stream)
    torch.cuda.synchronize()
    if use_ids:
        o["targets"] = targets
    assert bool((wide[:, c["tables"].shape[1]:] == -55).all())
    return {k: v.cpu().tolist() for k, v in o.items()}, tables.cpu().numpy()


def check(torch, c, **kw):
    got, tables = run(torch, c, **kw)
    want_tables = c["tables"].copy()
    want = ref.plan(c["cached"], c["fresh"], c["held"], c["page"], want_tables, c["free"], c["count"], c["ids"], c["room"])
    for k in got:
        assert got[k] == want[k], k
    assert np.array_equal(tables, want_tables)
    return got


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 511, 513, 2047, 2048, 2049, 4095, 4096, 4097, 9001])
@pytest.mark.parametrize("kind", ["decode", "mixed"])
def test_requests(gpu, n, kind):
    rng = np.random.default_rng(n)
    for page in (16, 1, 24):
        check(gpu, make(rng, n, page, kind, most_cached=60, most_fresh=9))


@pytest.mark.parametrize("page", [1, 2, 7, 16, 128, 100_000])
@pytest.mark.parametrize("held", [0, 3])
def test_pages(gpu, page, held):
    rng = np.random.default_rng(page)
    got = check(gpu, make(rng, 200, page, "mixed", held_over=held, most_cached=3 * page if page < 1000 else 500), stride_over=5)
    assert got["result"][0] >= 0


@pytest.mark.parametrize("zeros", [0.0, 0.9, 1.0])
def test_requests_without_tokens(gpu, zeros):
    rng = np.random.default_rng(5)
    for n in (1, 70, 4500):
        check(gpu, make(rng, n, 16, "mixed", zeros=zeros, room_over=0 if zeros < 1 else 3))


def test_long_requests(gpu):
    rng = np.random.default_rng(6)
    check(gpu, make(rng, 5, 64, "mixed", most_fresh=60_000, most_cached=100_000, zeros=0.0), use_ids=False)


@pytest.mark.parametrize("n", [3, 700, 2049])
def test_arrays_at_any_alignment(gpu, n):
    from paper_2607_29678_amd import step_plan

    torch = gpu
    c = make(np.random.default_rng(n), n, 16, "mixed", room_over=3)
    want_tables = c["tables"].copy()
    want = ref.plan(c["cached"], c["fresh"], None, 16, want_tables, c["free"], c["count"], c["ids"], c["room"])
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda")  # noqa: E731

    def off(k, t=torch.int32):  # one entry past an aligned address, with a guard behind
        return torch.full((k + 2,), -99, dtype=t, device="cuda")

    full = dict(offsets=off(n + 1), lengths=off(n), pages=off(n), slots=off(c["room"], torch.int64), positions=off(c["room"]),
                requests=off(c["room"]), targets=off(c["room"]), result=off(2, torch.int64))
    o = {k: v[1:-1] for k, v in full.items()}
    tables = dev(c["tables"])
    step_plan(dev(c["cached"]), dev(c["fresh"]), tables, dev(c["free"]), dev(np.array([c["count"]], dtype=np.int64)), 16,
              o["offsets"], o["lengths"], o["pages"], o["slots"], o["positions"], o["requests"], o["result"],
              ids=dev(c["ids"]), targets=o["targets"])
    torch.cuda.synchronize()
    for k in o:
        assert o[k].cpu().tolist() == want[k], k
        assert int(full[k][0]) == -99 and int(full[k][-1]) == -99
    assert np.array_equal(tables.cpu().numpy(), want_tables)


@pytest.mark.parametrize("room_over", [0, 1, 2, 3, 4, 5000])
def test_room_past_the_tokens(gpu, room_over):
    for n in (5, 2500):
        check(gpu, make(np.random.default_rng(room_over), n, 16, "mixed", room_over=room_over))


def test_no_requests(gpu):
    c = make(np.random.default_rng(7), 0, 16, "mixed", room_over=9)
    assert check(gpu, c)["result"][0] == 0


def test_slots_past_32_bits(gpu):
    c = make(np.random.default_rng(8), 40, 4096, "mixed", most_cached=20_000)
    c["free"] = c["free"] + np.int32(2**31 - 2**20 - 1)
    got = check(gpu, c)
    assert max(got["slots"]) > 2**40


def _broken():
    def case(**change):
        c = make(np.random.default_rng(9), 300, 16, "mixed", held_over=2, zeros=0.0)
        c.update({k: f(c) for k, f in change.items()})
        return c

    def at(name, value):
        def f(c):
            a = c[name].copy()
            a[137] = value
            return a
        return f

    yield "negative cached", case(cached=at("cached", -1)), -9
    yield "negative fresh", case(fresh=at("fresh", -5)), -9
    yield "negative held", case(held=at("held", -1)), -9
    yield "too wide", case(cached=at("cached", 16 * 1000)), -9
    yield "holds too many", case(held=at("held", 10**6)), -9
    yield "past 32 bits", case(cached=at("cached", 2**31 - 1), fresh=at("fresh", 2**31 - 1)), -9
    yield "more tokens than room", case(room=lambda c: c["room"] - 6, ids=lambda c: c["ids"][:-6]), -9
    yield "count past the list", case(count=lambda c: len(c["free"]) + 1), -9
    yield "negative count", case(count=lambda c: -1), -9
    yield "too few pages", case(count=lambda c: 3), -8


@pytest.mark.parametrize("name,c,code", list(_broken()), ids=[b[0] for b in _broken()])
def test_errors_that_the_device_finds(gpu, name, c, code):
    got = check(gpu, c)
    assert got["result"] == [code, c["count"]]


def test_errors_over_several_chunks(gpu):
    c = make(np.random.default_rng(10), 9001, 16, "mixed", most_cached=60, most_fresh=9)
    c["fresh"][8999] = -1
    assert check(gpu, c)["result"][0] == -9


def test_exactly_enough_pages(gpu):
    c = make(np.random.default_rng(11), 100, 16, "mixed")
    need = np.maximum(0, -(-(c["cached"] + c["fresh"]) // 16) - -(-c["cached"] // 16)).sum()
    c["count"] = int(need)
    assert check(gpu, c)["result"][1] == 0
    c["count"] -= 1
    assert check(gpu, c)["result"][0] == -8


def test_session_repair_keeps_pages(gpu):
    # 50 tokens in 4 pages; the repair keeps 33 and brings 20: position 33 lies in the third page, no new page
    c = dict(cached=np.array([33], np.int32), fresh=np.array([20], np.int32), held=np.array([4], np.int32), page=16,
             tables=np.array([[9, 4, 7, 2, -1]], np.int32), free=np.array([5, 6], np.int32), count=2,
             ids=np.arange(20, dtype=np.int32), room=20)
    got = check(gpu, c)
    assert got["slots"][0] == 7 * 16 + 1 and got["slots"][15] == 2 * 16 and got["pages"] == [4] and got["result"] == [20, 2]


def test_another_stream(gpu):
    s = gpu.cuda.Stream()
    c = make(np.random.default_rng(12), 500, 16, "mixed")
    gpu.cuda.synchronize()
    check(gpu, c, stream=s.cuda_stream)


def test_captured_step_on_new_lengths(gpu):
    """A captured plan follows the lengths that are in its arrays when it is replayed."""
    from paper_2607_29678_amd import step_plan

    torch = gpu
    rng = np.random.default_rng(13)
    n, page, room, width = 100, 16, 640, 40
    z = lambda k, t=torch.int32: torch.zeros(k, dtype=t, device="cuda")  # noqa: E731
    cached, fresh, ids, tables = z(n), z(n), z(room), z((n, width))
    free = torch.arange(5000, dtype=torch.int32, device="cuda")
    count = torch.tensor([5000], dtype=torch.int64, device="cuda")
    o = dict(offsets=z(n + 1), lengths=z(n), pages=z(n), slots=z(room, torch.int64), positions=z(room), requests=z(room),
             targets=z(room), result=z(2, torch.int64))

    def call(stream):
        step_plan(cached, fresh, tables, free, count, page, o["offsets"], o["lengths"], o["pages"], o["slots"],
                  o["positions"], o["requests"], o["result"], ids=ids, targets=o["targets"], stream=stream)

    g = torch.cuda.CUDAGraph()
    call(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call(torch.cuda.current_stream().cuda_stream)
    for _ in range(4):
        c = rng.integers(0, 300, n).astype(np.int32)
        f = rng.integers(0, 7, n).astype(np.int32)
        t0 = rng.integers(0, 1000, (n, width)).astype(np.int32)
        i = rng.integers(0, 50_000, room).astype(np.int32)
        for dst, src in ((cached, c), (fresh, f), (tables, t0), (ids, i)):
            dst.copy_(torch.from_numpy(src))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = ref.plan(c, f, None, page, t0, np.arange(5000), 5000, i, room)
        for k in o:
            assert o[k].cpu().tolist() == want[k], k
        assert np.array_equal(tables.cpu().numpy(), t0)
