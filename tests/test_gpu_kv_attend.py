"""Attention over pages on the GPU against its definition in 64 bits: lengths from none to thousands, odd groups and
strides, masks that leave rows empty, NaN and infinities where nobody looks, values out of range, streams and graphs."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv_support import Case  # noqa: E402

# (new tokens, tokens with them): one token; whole prompts; chunks; rows before the first key; nothing at all
MIX = [(1, 1), (1, 17), (0, 50), (5, 5), (3, 0), (4, 2), (130, 130), (1, 1000), (70, 333), (1, 128), (2, 129)]
DECODE = [(1, kv) for kv in (1, 2, 15, 16, 17, 31, 33, 64, 127, 128, 129, 255, 500, 1023, 2049)] + [(1, 0), (0, 9)]


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


def check(ctx, case, **opt):
    case.check(*case.run(ctx, **opt), **{k: v for k, v in opt.items() if k in ("scale", "causal", "window", "softcap")})
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("lens", [MIX, DECODE], ids=["mix", "decode"])
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,layout", [
    ("bf16", 128, 8, 2, 16, "dense"), ("fp16", 64, 8, 8, 32, "packed"), ("bf16", 64, 14, 2, 64, "heads_first"),
    ("fp16", 128, 5, 1, 128, "heads_first"), ("bf16", 128, 16, 1, 16, "packed"), ("fp16", 128, 40, 1, 32, "dense"),
    ("bf16", 64, 3, 3, 16, "dense"), ("bf16", 128, 12, 2, 64, "dense"), ("fp16", 64, 8, 4, 128, "packed"),
    ("bf16", 64, 32, 1, 128, "dense")])
def test_types_heads_and_layouts(ctx, lens, dtype, D, Hq, Hkv, page, layout):
    check(ctx, Case(lens, dtype, D, Hq, Hkv, page, seed=D + Hq, layout=layout))


@pytest.mark.parametrize("lens", [MIX, DECODE], ids=["mix", "decode"])
@pytest.mark.parametrize("opt", [dict(causal=False), dict(window=1), dict(window=7), dict(window=130), dict(softcap=5.0),
                                 dict(softcap=30.0, window=64), dict(softcap=800.0), dict(softcap=0.01), dict(scale=0.5), dict(scale=-0.1), dict(scale=0.0)],
                         ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
def test_masks_caps_and_scales(ctx, lens, opt):
    check(ctx, Case(lens, "bf16", 64, 8, 2, 16, seed=5), **opt)
    check(ctx, Case(lens, "fp16", 128, 6, 3, 32, seed=6), **opt)


@pytest.mark.parametrize("lens", [[(1, 20011)], [(2, 30000), (1, 5), (1, 9000)], [(300, 9001)], [(1, 4096)] * 3, [(2000, 2000)],
                                  [(513, 513), (100, 5000), (1, 1), (17, 40)], [(1, 300)] * 200, [(9, 200)] * 33],
                         ids=lambda x: "_".join(f"{q}of{kv}" for q, kv in x[:3]) + f"x{len(x)}")
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", [("bf16", 128, 8, 2, 16), ("fp16", 64, 16, 4, 64), ("bf16", 128, 7, 1, 128)])
def test_lengths_that_are_split_and_joined(ctx, lens, dtype, D, Hq, Hkv, page):
    case = Case(lens, dtype, D, Hq, Hkv, page, seed=9)
    check(ctx, case)
    a, b = case.run(ctx), case.run(ctx)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])  # the order of sums is fixed


@pytest.mark.parametrize("scores", [6.0, 40.0])
@pytest.mark.parametrize("lens", [[(1, 3000), (1, 77)], [(200, 1500), (3, 900)]], ids=["decode", "chunk"])
def test_scores_far_apart(ctx, lens, scores):
    """Running maxima that grow by hundreds on the way."""
    for dtype, D in (("bf16", 128), ("fp16", 64)):
        case = Case(lens, dtype, D, 8, 2, 16, seed=3, scores=scores)
        for b, (_, kv) in enumerate(lens):  # ascending towards the end
            k = case.keys[b] * torch.linspace(0.1, 1, kv, device="cuda")[:, None, None].to(case.dt)
            case.keys[b] = k
            case.set(b, k, case.values[b])
        check(ctx, case)


@pytest.mark.parametrize("where", ["future", "window"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("q", [1, 2, 5, 40, 300])
def test_what_a_row_does_not_see_does_not_matter(ctx, where, value, q):
    """Keys and values of NaN or infinity at a position that some rows of a request see and others do not: the ones
    that do not are as if it were not there."""
    kv, opt = 700, dict(window=200) if where == "window" else {}
    case = Case([(q, kv), (1, 90)], "bf16", 128, 8, 2, 16, seed=q)
    k, v = case.keys[0].clone(), case.values[0].clone()
    # seen by the last row alone (the new token itself), or by the first rows at most
    at = kv - 1 if where == "future" else kv - q - 199 - 1 + (1 if q > 1 else 0)
    v[at, :, ::7] = value
    if value != value:
        k[at] = value
    case.set(0, k, v)
    out, lse = case.run(ctx, **opt)
    kvdro.kvdro_sync(ctx)
    p = np.arange(kv - q, kv)
    sees = (p >= at) & ((p - at) < 200 if where == "window" else True)
    T = case.T - 1
    blind = torch.from_numpy(np.nonzero(~sees)[0]).cuda()
    clean = Case([(q, kv), (1, 90)], "bf16", 128, 8, 2, 16, seed=q)
    want, wz = clean.run(ctx, **opt)
    assert torch.isfinite(out[blind]).all()
    clean.check(torch.where(torch.from_numpy(np.concatenate([sees, [False]])).cuda()[:, None, None], want, out),
                torch.where(torch.from_numpy(np.concatenate([sees, [False]])).cuda()[:, None], wz, lse), **opt)
    seers = out[:T][torch.from_numpy(np.nonzero(sees)[0]).cuda()]
    if len(seers):
        hit = seers[..., ::7]
        assert torch.isnan(hit).all() if value != value else (hit == value).all()
        if value == value:  # the other components are what they would be
            other = torch.ones(128, dtype=torch.bool)
            other[::7] = False
            assert torch.isfinite(seers[..., other]).all()


def test_infinite_values_that_every_row_sees(ctx):
    case = Case([(1, 300), (50, 400)], "bf16", 128, 8, 2, 16, seed=2)
    for b in range(2):
        v = case.values[b].clone()
        v[3, :, 5] = float("inf")
        case.set(b, case.keys[b], v)
    out, _ = case.run(ctx)
    assert (out[..., 5] == float("inf")).all()
    keep = [d for d in range(128) if d != 5]
    assert torch.isfinite(out[..., keep]).all()


def test_out_of_range_pages_are_left_out_and_reported(ctx):
    for lens in ([(1, 100), (1, 200), (1, 40)], [(60, 100), (150, 200), (30, 40)]):
        case = Case(lens, "bf16", 128, 8, 2, 16, seed=4)
        for bad in (-1, 10 ** 6):
            table = case.table.clone()
            case.table[1, 3] = bad
            out, lse = case.run(ctx)
            with pytest.raises(kvdro.KvdroError) as e:
                kvdro.kvdro_sync(ctx)
            assert e.value.status == kvdro.KVDRO_ERANGE
            case.check(out, lse, only=(0, 2))
            case.table = table
        case.kv_len[1] = 10 ** 6  # more than the table's row holds: no keys
        out, lse = case.run(ctx)
        with pytest.raises(kvdro.KvdroError):
            kvdro.kvdro_sync(ctx)
        t0, t1 = case.off[1], case.off[2]
        assert (out[t0:t1] == 0).all() and (lse[t0:t1] == float("-inf")).all()
        case.check(out, lse, only=(0, 2))


def test_tokens_of_no_request_and_outputs_inside_their_extents(ctx):
    case = Case([(3, 50), (1, 70)], "fp16", 64, 6, 2, 16, seed=8)
    T, H, D = case.T + 5, 6, 64
    q = torch.randn((T, H, D), device="cuda").to(case.dt)
    q[:case.T] = case.q
    store = torch.full((T + 2, H + 1, D + 8), 55.0, dtype=case.dt, device="cuda")
    out = store[1:-1, :H, :D]
    lse = torch.full((T + 2, H), 55.0, device="cuda")
    cache = kvdro.kvdro_kv_open(ctx, case.k, case.v)
    for max_q in (0, 1, 3, 1000):
        kvdro.kvdro_kv_attend(cache, q, case.q_off, case.kv_len, case.table, out, lse=lse[1:-1], max_q=max_q)
        kvdro.kvdro_sync(ctx)
        case.check(out[:case.T], lse[1:case.T + 1])
        assert (out[case.T:] == 0).all() and (lse[case.T + 1:-1] == float("-inf")).all()
        guard = store.clone()
        guard[1:-1, :H, :D] = 55.0
        assert (guard == 55.0).all() and (lse[0] == 55).all() and (lse[-1] == 55).all()
    # fewer tokens than the requests have: the rest is left out
    out = torch.full((2, H, D), 55.0, dtype=case.dt, device="cuda")
    kvdro.kvdro_kv_attend(cache, q[:2], case.q_off, case.kv_len, case.table, out)
    full, _ = case.run(ctx)
    assert torch.equal(out, full[:2])
    kvdro.kvdro_kv_close(cache)


def test_hints_streams_and_graphs_change_nothing(ctx):
    for lens in (MIX, DECODE):
        case = Case(lens, "bf16", 128, 8, 2, 16, seed=12)
        want = case.run(ctx)
        for max_q in (0, 1, 7, 100000):
            case.check(*case.run(ctx, max_q=max_q))
        other = torch.cuda.Stream()
        got = case.run(ctx, stream=other)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        # calls on two streams share the context's scratch
        big = Case([(1, 20000)] if lens is DECODE else [(300, 4000)], "bf16", 128, 8, 2, 16, seed=1)
        cache, bc = kvdro.kvdro_kv_open(ctx, case.k, case.v), kvdro.kvdro_kv_open(ctx, big.k, big.v)
        outs = [[torch.empty_like(c.q) for _ in range(4)] for c in (case, big)]
        torch.cuda.synchronize()
        for i in range(4):
            kvdro.kvdro_kv_attend(bc, big.q, big.q_off, big.kv_len, big.table, outs[1][i], stream=other)
            kvdro.kvdro_kv_attend(cache, case.q, case.q_off, case.kv_len, case.table, outs[0][i], stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        for c, o in ((case, outs[0]), (big, outs[1])):
            assert all(torch.equal(x, o[0]) for x in o)
            c.check(o[0], None)
        graph = torch.cuda.CUDAGraph()
        out, lse = torch.zeros_like(case.q), torch.zeros((case.T, 8), device="cuda")
        with torch.cuda.graph(graph):
            kvdro.kvdro_kv_attend(cache, case.q, case.q_off, case.kv_len, case.table, out, lse=lse, stream=torch.cuda.current_stream())
        for _ in range(2):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            case.check(out, lse)
    kvdro.kvdro_sync(ctx)


def test_offsets_past_32_bits(ctx):
    """Pages 2^28 elements apart: the last ones lie past 2^32 elements."""
    n, page, Hkv, D = 18, 16, 2, 64
    case = Case([(1, 200), (2, 60)], "bf16", D, 4, Hkv, page, seed=3, spare=1)
    store = torch.empty((n - 1) * (1 << 28) + 2 * page * Hkv * D, dtype=torch.bfloat16, device="cuda")
    k, v = (store.as_strided((n, page, Hkv, D), (1 << 28, Hkv * D, D, 1), i * page * Hkv * D) for i in range(2))
    assert case.k.shape == k.shape
    for i in range(n):
        k[i], v[i] = case.k[i], case.v[i]
    case.k, case.v = k, v
    check(ctx, case)


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 4, 1), ("fp16", 64, 6, 2)])
@pytest.mark.parametrize("max_q", [1, 0])
def test_many_requests(ctx, dtype, D, Hq, Hkv, max_q):
    """More requests than threads, so that a thread counts several; some with more row tiles than it counts by itself."""
    rng = np.random.default_rng(D)
    lens = [(int(rng.integers(0, 4)), int(rng.integers(0, 60))) for _ in range(1500)]
    for b, n in ((3, 900), (700, 2100), (1499, 400)):
        lens[b] = (n if max_q == 0 else 30, n + 100)
    case = Case(lens, dtype, D, Hq, Hkv, 16, seed=1)
    out, lse = case.run(ctx, max_q=max_q)
    case.check(out, lse, only=set(range(0, 1500, 23)) | {3, 700, 1499})
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("skip", [0, 1, 2, 5, 6])
@pytest.mark.parametrize("lens", [[(1, 9000)] * 40, [(300, 4000)] * 6, [(1, 9000)] * 20 + [(300, 4000)] * 4], ids=["decode", "chunk", "both"])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(monkeypatch, ctx, skip, lens):
    """Failure detection without a fault: every CTA leaves one copy out, so nothing completes its barrier, and the
    bounded wait for it (1 ms under the hook) gives up."""
    case = Case(lens, "bf16", 128, 8, 2, 16, seed=1)
    monkeypatch.setenv("KVDRO_TEST_SKIP_CHUNK", str(skip))
    broken = kvdro.kvdro_create(0)
    monkeypatch.delenv("KVDRO_TEST_SKIP_CHUNK")
    try:
        for _ in range(2):
            case.run(broken)
            with pytest.raises(kvdro.KvdroError) as e:
                kvdro.kvdro_sync(broken)
            assert e.value.status == kvdro.KVDRO_ETIMEOUT
        kvdro.kvdro_sync(broken)
    finally:
        kvdro.kvdro_destroy(broken)
    case.check(*case.run(ctx), only={0, len(lens) - 1})
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("n", [1, 2, 3])
def test_injected_allocation_failure_reports_enomem(monkeypatch, n):
    monkeypatch.setenv("KVDRO_TEST_FAIL_ALLOC", str(n))
    c = kvdro.kvdro_create(0)
    k = torch.zeros((2, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    try:
        caches = []
        try:
            caches.append(kvdro.kvdro_kv_open(c, k, k.clone()))
        except kvdro.KvdroError as e:
            assert e.status == kvdro.KVDRO_ENOMEM
        caches.append(kvdro.kvdro_kv_open(c, k, k.clone()))  # the next try allocates what is missing
        q = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
        i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        out = torch.ones_like(q)
        kvdro.kvdro_kv_attend(caches[-1], q, i(0, 1), i(5), i(1)[None], out)
        kvdro.kvdro_sync(c)
        assert (out == 0).all()
    finally:
        kvdro.kvdro_destroy(c)
    with pytest.raises(ValueError, match="closed"):
        kvdro.kvdro_kv_attend(caches[-1], q, i(0, 1), i(5), i(1)[None], out)
