"""Page cache calls on several streams: scratch, status and what kvdro_sync waits for."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv_support import Case  # noqa: E402

A_WHILE = 500_000_000  # GPU clocks: a quarter of a second


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("lens", [[(1, 20000), (1, 300)], [(300, 4000)], [(1, 9000), (300, 3000)]], ids=["decode", "chunk", "both"])
def test_scratch_of_a_new_context_is_clear_whatever_stream_uses_it_first(lens):
    """The default stream is busy when the cache is opened, and the first call, whose rows are split over many CTAs,
    goes to a stream that is not ordered behind it."""
    case = Case(lens, "bf16", 128, 8, 2, 16, seed=1)
    first = kvdro.kvdro_create(0)  # loads the kernels
    case.check(*case.run(first))
    kvdro.kvdro_destroy(first)
    side = torch.cuda.Stream()
    for _ in range(3):
        junk = torch.full((1 << 20,), 7, dtype=torch.int32, device="cuda")  # what fresh memory may hold
        del junk
        torch.cuda.empty_cache()
        ctx = kvdro.kvdro_create(0)
        try:
            torch.cuda.synchronize()
            torch.cuda._sleep(A_WHILE)
            cache = kvdro.kvdro_kv_open(ctx, case.k, case.v)
            busy = not torch.cuda.default_stream().query()
            outs = [torch.empty_like(case.q) for _ in range(4)]
            for out in outs:
                kvdro.kvdro_kv_attend(cache, case.q, case.q_off, case.kv_len, case.table, out, stream=side)
            side.synchronize()
            assert busy, "opening a cache waited for the caller's work"
            for out in outs:
                case.check(out, None)
            kvdro.kvdro_sync(ctx)
        finally:
            kvdro.kvdro_destroy(ctx)


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def small_plan(ctx, stream=None):
    a = [ints(0), ints(1), ints(0), ints(-1)[None], ints(0, 1), ints(0, 2), ints(0), ints(0, 0), ints(0, 0), ints(0), ints(0)]
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    kvdro.kvdro_kv_plan(ctx, 16, *a, stream=stream)
    return a


def test_sync_waits_for_a_grid_call_on_another_stream():
    ctx = kvdro.kvdro_create(0)
    try:
        kvdro.kvdro_load_samples(ctx, 1, np.array([0, 100]), np.arange(100, dtype=np.int32), np.array([100], np.int32), None)
        r, side = np.arange(10, dtype=np.int32), torch.cuda.Stream()
        cost = torch.zeros((1, 1, 1, 10), dtype=torch.float64, device="cuda")

        def grid(stream):
            kvdro.kvdro_eval_dual(ctx, 10, r, 1, [1.0], 1, [10.0], [1.0], cost=cost, stream=stream)
        grid(side)
        want = cost.clone()
        small_plan(ctx)
        kvdro.kvdro_sync(ctx)
        cost.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(A_WHILE)
        grid(side)
        small_plan(ctx)
        kvdro.kvdro_sync(ctx)
        assert side.query()
        assert torch.equal(cost, want)
    finally:
        kvdro.kvdro_destroy(ctx)


def test_sync_waits_for_the_last_attention_on_another_stream():
    case = Case([(1, 9000)] * 4, "bf16", 128, 8, 2, 16, seed=1)
    ctx, side = kvdro.kvdro_create(0), torch.cuda.Stream()
    try:
        case.check(*case.run(ctx, stream=side))
        cache, out = kvdro.kvdro_kv_open(ctx, case.k, case.v), torch.empty_like(case.q)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(A_WHILE)
        kvdro.kvdro_kv_attend(cache, case.q, case.q_off, case.kv_len, case.table, out, stream=side)
        small_plan(ctx)
        kvdro.kvdro_sync(ctx)
        assert side.query()
        case.check(out, None)
    finally:
        kvdro.kvdro_destroy(ctx)


def test_reports_are_neither_lost_nor_repeated():
    """Bad slots on a side stream at about the time when another stream's report is taken."""
    ctx, side = kvdro.kvdro_create(0), torch.cuda.Stream()
    k = torch.zeros((2, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    bad, new = ints(32), torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")

    def reports():
        try:
            kvdro.kvdro_sync(ctx)
        except kvdro.KvdroError as e:
            assert e.status == kvdro.KVDRO_ERANGE
            return True
        return False
    try:
        cache = kvdro.kvdro_kv_open(ctx, k, k.clone())
        torch.cuda.synchronize()
        for i in range(100):
            with torch.cuda.stream(side):
                torch.cuda._sleep(1 + 500 * i)
            kvdro.kvdro_kv_append(cache, new, new, bad, stream=side)
            late = not side.query()
            kvdro.kvdro_kv_append(cache, new, new, bad)
            assert reports(), i
            late &= not side.query()
            side.synchronize()
            assert reports() or not late, i
            assert not reports(), i
    finally:
        kvdro.kvdro_destroy(ctx)


def test_scratch_is_clear_after_a_wait_that_ran_out(monkeypatch):
    """A context whose kernels leave out every CTA's 31st copy: a large call runs out of its wait, small ones do not come
    that far.  They follow at once, on the same stream and on others, their rows split over many CTAs."""
    big, small = (Case(lens, "bf16", 64, 4, 2, 16, seed=1) for lens in ([(1, 20000)] * 60, [(1, 20000)]))
    monkeypatch.setenv("KVDRO_TEST_SKIP_CHUNK", "30")
    ctx = kvdro.kvdro_create(0)
    monkeypatch.delenv("KVDRO_TEST_SKIP_CHUNK")
    streams = [torch.cuda.Stream() for _ in range(2)]
    try:
        caches = [kvdro.kvdro_kv_open(ctx, c.k, c.v) for c in (big, small)]
        out, outs = torch.empty_like(big.q), [torch.empty_like(small.q) for _ in range(8)]
        torch.cuda.synchronize()
        for _ in range(3):
            kvdro.kvdro_kv_attend(caches[0], big.q, big.q_off, big.kv_len, big.table, out, stream=streams[0], max_q=1)
            small_plan(ctx)
            with pytest.raises(kvdro.KvdroError) as e:
                kvdro.kvdro_sync(ctx)
            assert e.value.status == kvdro.KVDRO_ETIMEOUT
            for i, o in enumerate(outs):
                kvdro.kvdro_kv_attend(caches[1], small.q, small.q_off, small.kv_len, small.table, o, stream=streams[i % 2], max_q=1)
            kvdro.kvdro_sync(ctx)
            torch.cuda.synchronize()
            for o in outs:
                small.check(o, None)
    finally:
        kvdro.kvdro_destroy(ctx)


def step(cache, ctx, new, out, stream=None):
    """A plan for one request of 40 tokens, the write, the attention, with no stream named."""
    a = {"cached": ints(0), "new_len": ints(40), "held": ints(0), "table": ints(-1, -1, -1)[None], "ring": ints(2, 0, 1), "pool": ints(0, 3),
         "held_out": ints(0), "pool_out": ints(0, 0), "q_off": ints(0, 0), "kv_len": ints(0), "slot": torch.full_like(ints(*range(40)), -1)}

    def go():
        kvdro.kvdro_kv_plan(ctx, 16, **a, stream=stream)
        kvdro.kvdro_kv_append(cache, new[:, :1], new[:, 1:], a["slot"], stream=stream)
        kvdro.kvdro_kv_attend(cache, new[:, :1], a["q_off"], a["kv_len"], a["table"], out, max_q=40, stream=stream)
    return go


def test_calls_go_to_torchs_current_stream():
    """Behind work of the current stream that fills what they read, and in a graph that is captured on it."""
    ctx, side = kvdro.kvdro_create(0), torch.cuda.Stream()
    g = torch.Generator(device="cuda").manual_seed(1)
    try:
        k, v = (torch.zeros((3, 16, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache = kvdro.kvdro_kv_open(ctx, k, v)
        data = torch.randn((40, 2, 64), generator=g, device="cuda").bfloat16()
        want, out, new = (torch.zeros((40, n, 64), dtype=torch.bfloat16, device="cuda") for n in (1, 1, 2))
        new.copy_(data)
        step(cache, ctx, new, want)()
        kvdro.kvdro_sync(ctx)
        assert want.abs().max() > 0
        new.zero_()
        go = step(cache, ctx, new, out)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(A_WHILE)
            new.copy_(data)
            go()
            assert not side.query() and torch.cuda.default_stream().query()
        side.synchronize()
        kvdro.kvdro_sync(ctx)
        assert torch.equal(out, want)
        graph, new2, out2 = torch.cuda.CUDAGraph(), data.clone(), torch.zeros_like(out)
        go = step(cache, ctx, new2, out2)
        with torch.cuda.graph(graph):
            go()
        new2.copy_(data.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        step(cache, ctx, new2, want)()
        assert torch.equal(out2, want)
        kvdro.kvdro_sync(ctx)
        # a stream that is named is the one that is used
        out.zero_()
        go = step(cache, ctx, new2, out, stream=torch.cuda.default_stream())
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(A_WHILE)
            go()
            torch.cuda.default_stream().synchronize()
            assert not side.query()
        assert torch.equal(out, want)
    finally:
        kvdro.kvdro_destroy(ctx)


def test_a_call_that_gave_up_leaves_its_neighbours_alone(monkeypatch):
    """Chunks whose waits run out, many times, beside another context's calls on the same SMs: what was still on its way
    when a CTA gave up does not land in the next one's memory."""
    lens = [(60, 300), (40, 3000), (300, 500), (200, 200), (20, 90)] * 6
    case = Case(lens, "bf16", 128, 8, 2, 16, seed=1)
    monkeypatch.setenv("KVDRO_TEST_SKIP_CHUNK", "0")
    broken = kvdro.kvdro_create(0)
    monkeypatch.delenv("KVDRO_TEST_SKIP_CHUNK")
    ctx, sides = kvdro.kvdro_create(0), [torch.cuda.Stream() for _ in range(2)]
    try:
        want = torch.empty_like(case.q)
        caches = [kvdro.kvdro_kv_open(c, case.k, case.v) for c in (broken, ctx)]
        kvdro.kvdro_kv_attend(caches[1], case.q, case.q_off, case.kv_len, case.table, want, max_q=300)
        case.check(want, None, only={0, 3, 29})
        junk, outs = torch.empty_like(want), [torch.zeros_like(want) for _ in range(30)]
        torch.cuda.synchronize()
        for out in outs:
            kvdro.kvdro_kv_attend(caches[0], case.q, case.q_off, case.kv_len, case.table, junk, max_q=300, stream=sides[0])
            kvdro.kvdro_kv_attend(caches[1], case.q, case.q_off, case.kv_len, case.table, out, max_q=300, stream=sides[1])
        with pytest.raises(kvdro.KvdroError) as e:
            kvdro.kvdro_sync(broken)
        assert e.value.status == kvdro.KVDRO_ETIMEOUT
        kvdro.kvdro_sync(ctx)
        assert all(torch.equal(out, want) for out in outs)
    finally:
        kvdro.kvdro_destroy(broken)
        kvdro.kvdro_destroy(ctx)
