"""Calls on caches of 8 bits and shared prefixes beyond single ones: waits that run out, other streams, graphs, many requests, far offsets."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv8_support import E4M3, F64, Case8, Shared, arrays, quantise, two  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


@pytest.mark.parametrize("skip", [0, 1, 2, 5])
@pytest.mark.parametrize("kind", ["decode", "chunk", "both", "shared", "each"])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(monkeypatch, ctx, kind, skip):
    """Every CTA leaves one copy out, so nothing completes its barrier, and the bounded wait for it (1 ms under the hook) gives up."""
    if kind in ("shared", "each"):
        case = Shared([(1, 9000)] * 40, [0, 40], [20000 if kind == "shared" else 3000], bits=8, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=1)
    else:
        case = Case8({"decode": [(1, 9000)] * 40, "chunk": [(300, 4000)] * 6, "both": [(1, 9000)] * 20 + [(300, 4000)] * 4}[kind], "bf16", 128,
                     8, 2, 16, seed=1)
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
    if kind in ("shared", "each"):
        case.check(*case.run(ctx))
    else:
        case.check(*case.run(ctx), only={0, len(case.lens) - 1})
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("lens", [[(1, 700), (1, 9000)], [(200, 900), (1, 40)]], ids=["decode", "chunk"])
def test_streams_and_graphs(ctx, lens):
    """Calls on two streams that share a context's scratch, and a graph whose queries change."""
    case, big = Case8(lens, "bf16", 128, 8, 2, 16, seed=1), Case8([(1, 30000)] * 3, "bf16", 128, 8, 2, 16, seed=2)
    cache, bc, other = case.open(ctx), big.open(ctx), torch.cuda.Stream()
    outs = [[torch.empty_like(c.q) for _ in range(4)] for c in (case, big)]
    torch.cuda.synchronize()
    for i in range(4):
        kvdro.kvdro_kv_attend(bc, big.q, big.q_off, big.kv_len, big.table, outs[1][i], stream=other)
        kvdro.kvdro_kv_attend(cache, case.q, case.q_off, case.kv_len, case.table, outs[0][i])
    torch.cuda.synchronize()
    for c, o in ((case, outs[0]), (big, outs[1])):
        assert all(torch.equal(x, o[0]) for x in o)
        c.check(o[0], None)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(case.q)
    with torch.cuda.graph(graph):
        kvdro.kvdro_kv_attend(cache, case.q, case.q_off, case.kv_len, case.table, out)
    for seed in (3, 4):
        case.q.copy_(torch.randn(case.q.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        case.check(out, None)
    kvdro.kvdro_sync(ctx)


def test_a_step_in_a_graph(ctx):
    """Write, attend and read of new rows in one graph, on a stream that is not the default one."""
    n, page, heads, D, T, i32 = 30, 16, 2, 128, 40, dict(dtype=torch.int32, device="cuda")
    k, v = arrays(n, page, heads, D, "dense")
    exps = [torch.ones((n, heads, page), dtype=torch.uint8, device="cuda") for _ in "kv"]
    cache = kvdro.kvdro_kv_open8(ctx, k.view(E4M3), v.view(E4M3), *exps, torch.bfloat16)
    table, q_off, kv_len = torch.tensor([[3, 7, 1]], **i32), torch.tensor([0, T], **i32), torch.tensor([T], **i32)
    slot = table[0].repeat_interleave(page)[:T] * page + torch.arange(T, **i32) % page
    qkv = torch.empty((T, 4 * heads, D), dtype=torch.bfloat16, device="cuda")
    q, kn, vn = qkv[:, :2 * heads], qkv[:, 2 * heads:3 * heads], qkv[:, 3 * heads:]
    out, got = torch.empty((T, 2 * heads, D), dtype=torch.bfloat16, device="cuda"), torch.empty((2, T, heads, D), dtype=torch.bfloat16, device="cuda")

    def step():
        kvdro.kvdro_kv_append(cache, kn, vn, slot)
        kvdro.kvdro_kv_attend(cache, q, q_off, kv_len, table, out, max_q=T)
        kvdro.kvdro_kv_read(cache, q_off, kv_len, table, got[0], got[1])

    qkv.normal_()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
    for seed in (1, 2):
        torch.cuda.synchronize()
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        held = []
        for rows, x in ((kn, got[0]), (vn, got[1])):
            c, e = quantise(rows)
            held.append(c * two(e)[..., None])
            assert torch.equal(x.to(F64), held[-1])
        kk, vv = (x.repeat_interleave(2, 1) for x in held)
        s = torch.einsum("thd,jhd->htj", q.double(), kk) / D ** 0.5
        s = s.masked_fill(torch.arange(T, device="cuda")[None] > torch.arange(T, device="cuda")[:, None], float("-inf"))
        w = torch.softmax(s, -1)
        ref, size = (torch.einsum("htj,jhd->thd", w, x) for x in (vv, vv.abs()))
        assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12) * size).all()
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 4, 1), ("fp16", 64, 6, 2)])
@pytest.mark.parametrize("max_q", [1, 0])
def test_many_requests(ctx, dtype, D, Hq, Hkv, max_q):
    rng = np.random.default_rng(D)
    lens = [(int(rng.integers(0, 4)), int(rng.integers(0, 60))) for _ in range(1500)]
    for b, n in ((3, 900), (700, 2100), (1499, 400)):
        lens[b] = (n if max_q == 0 else 30, n + 100)
    case = Case8(lens, dtype, D, Hq, Hkv, 16, seed=1)
    out, lse = case.run(ctx, max_q=max_q)
    case.check(out, lse, only=set(range(0, 1500, 23)) | {3, 700, 1499})
    kvdro.kvdro_sync(ctx)


def test_many_prefixes(ctx):
    """Three hundred of them, some without tokens, some without requests."""
    rng = np.random.default_rng(3)
    lens = [(int(rng.integers(1, 4)), int(rng.integers(3, 30))) for _ in range(500)]
    share = np.sort(rng.integers(0, 501, 301)).tolist()
    prefixes = [int(x) for x in rng.integers(0, 90, 300)]
    for bits in (16, 8):
        for wide in (False, True):
            s = Shared(lens, share, prefixes, bits=bits, wide=wide, dtype="bf16", D=64, Hq=4, Hkv=2, page=16, seed=4)
            out, lse = s.run(ctx)
            whole = s.whole()
            type(s.c).check(whole, out, lse, only=set(range(0, len(whole.lens), 17)))
            kvdro.kvdro_sync(ctx)


def test_offsets_past_32_bits(ctx):
    """Pages 2^28 bytes apart: the last ones lie past 2^32 bytes, for single tokens, chunks, writes and reads."""
    page, Hkv, D = 16, 2, 64
    for lens in ([(1, 200), (2, 60)], [(40, 200), (2, 60)]):
        case = Case8(lens, "bf16", D, 4, Hkv, page, seed=3)
        count = case.codes[0].shape[0]
        store = torch.empty((count - 1) * (1 << 28) + 2 * page * Hkv * D, dtype=torch.uint8, device="cuda")
        far = [store.as_strided((count, page, Hkv, D), (1 << 28, Hkv * D, D, 1), i * page * Hkv * D) for i in range(2)]
        for i in range(count):
            far[0][i], far[1][i] = case.codes[0][i], case.codes[1][i]
        case.codes = far
        assert (count - 1) << 28 >= 1 << 32
        case.check(*case.run(ctx))
        cache = case.open(ctx)
        k, v = (torch.empty((case.T, Hkv, D), dtype=case.dt, device="cuda") for _ in "kv")
        kvdro.kvdro_kv_read(cache, case.q_off, case.kv_len, case.table, k, v)
        slot = case.table[0, 12:13].repeat_interleave(case.T) * page + torch.arange(case.T, dtype=torch.int32, device="cuda") % page
        kvdro.kvdro_kv_append(cache, k[:1], v[:1], slot[:1])
        kvdro.kvdro_sync(ctx)
        t = case.off[1] - 1
        assert torch.equal(k[t].to(F64), case.keys[0][-1]) and torch.equal(v[t].to(F64), case.values[0][-1])
        c, _ = quantise(k[:1])
        p = int(case.table[0, 12])
        assert torch.equal(far[0][p, 0].view(E4M3).to(F64), c[0])
        kvdro.kvdro_kv_close(cache)


def test_values_beyond_fp16_and_scales_of_zero(ctx):
    """A cache that was written as BF16 and is opened as FP16: values beyond its range are infinities, for the rows that see them.  A scale
    byte of 0 stands for zeros."""
    for q in (1, 60):
        case = Case8([(q, 100), (1, 50)], "bf16", 64, 2, 1, 16, seed=q)
        v = case.values[0].to(case.dt)
        v[99, :, 3] = 3.0e5  # seen by the last row alone
        case.set(0, case.keys[0].to(case.dt), v)
        case.dt, case.q = torch.float16, case.q.to(torch.float16)
        out, _ = case.run(ctx)
        last = out[q - 1]
        rest = torch.ones(64, dtype=torch.bool)
        rest[3] = False
        assert torch.isfinite(out[:q - 1]).all() and torch.isfinite(last[:, rest]).all()
        if q > 1:  # widened on the way to the tiles; single tokens multiply codes, and 3e5 times a small weight may be finite
            assert torch.isinf(last[:, 3]).all()
        k = torch.empty((case.T, 1, 64), dtype=torch.float16, device="cuda")
        got = torch.empty_like(k)
        cache = case.open(ctx)
        kvdro.kvdro_kv_read(cache, case.q_off, case.kv_len, case.table, k, got)
        assert torch.isinf(got[q - 1, 0, 3]) and torch.isfinite(got[:q - 1]).all()
        case.exps[0].zero_()  # keys of zeros: the mean of the values
        case.exps[1].fill_(127)
        out, lse = case.run(ctx)
        kvdro.kvdro_kv_close(cache)
        mean = case.codes[1][case.places(1, 50)].view(E4M3).to(F64).mean(0)
        assert ((out[-1].to(F64) - mean).abs() <= 2.0 ** -10 * 448).all()
        assert ((lse[-1] - np.log(50)).abs() < 1e-5).all()
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("n", [1, 2, 3])
def test_injected_allocation_failure_reports_enomem(monkeypatch, n):
    monkeypatch.setenv("KVDRO_TEST_FAIL_ALLOC", str(n))
    c = kvdro.kvdro_create(0)
    k, e = torch.zeros((2, 16, 1, 64), dtype=torch.float8_e4m3fn, device="cuda"), torch.ones((2, 1, 16), dtype=torch.uint8, device="cuda")
    try:
        caches = []
        try:
            caches.append(kvdro.kvdro_kv_open8(c, k, k.clone(), e, e.clone(), torch.float16))
        except kvdro.KvdroError as x:
            assert x.status == kvdro.KVDRO_ENOMEM
        caches.append(kvdro.kvdro_kv_open8(c, k, k.clone(), e, e.clone(), torch.float16))
        out = torch.ones((3, 1, 64), dtype=torch.float16, device="cuda")
        i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        kvdro.kvdro_kv_read(caches[-1], i(0, 3), i(5), i(1)[None], out, out.clone())
        kvdro.kvdro_sync(c)
        assert (out == 0).all()
    finally:
        kvdro.kvdro_destroy(c)
    with pytest.raises(ValueError, match="closed"):
        kvdro.kvdro_kv_read(caches[-1], i(0, 3), i(5), i(1)[None], out, out.clone())


def test_refusals(ctx):
    def dev(*shape, dt=torch.float8_e4m3fn):
        return torch.zeros(shape, dtype=torch.uint8 if dt is torch.float8_e4m3fn else dt, device="cuda").view(dt)

    opened, e = kvdro.kvdro_kv_open8, dev(2, 1, 16, dt=torch.uint8)
    k = dev(2, 16, 1, 64)
    for args, match in (((k, k, e[:1], e, torch.bfloat16), "k_exp"), ((k, k, e, e.transpose(1, 2), torch.bfloat16), "v_exp"),
                        ((k, dev(2, 16, 2, 64), e, e, torch.bfloat16), "differ"), ((dev(2, 16, 64, 2).transpose(2, 3),) * 2 + (e, e, torch.bfloat16), "contiguous")):
        with pytest.raises(ValueError, match=match):
            opened(ctx, *args)
    for args, match in (((k, k, e.to(torch.int32), e, torch.bfloat16), "k_exp"), ((k.view(torch.uint8), k, e, e, torch.bfloat16), "k:"),
                        ((k, k, e, e, torch.float32), "dtype")):
        with pytest.raises(TypeError, match=match):
            opened(ctx, *args)

    def refused(call, *a, match="", **kw):
        with pytest.raises(kvdro.KvdroError, match=match) as x:
            call(*a, **kw)
        assert x.value.status == kvdro.KVDRO_EINVAL

    refused(opened, ctx, dev(2, 24, 1, 64), dev(2, 24, 1, 64), dev(2, 1, 24, dt=torch.uint8), dev(2, 1, 24, dt=torch.uint8), torch.bfloat16, match="page_size")
    refused(opened, ctx, dev(2, 16, 1, 96), dev(2, 16, 1, 96), e, e, torch.bfloat16, match="head_dim")
    odd = dev(2, 16, 2, 72)
    two_heads = dev(2, 2, 16, dt=torch.uint8)
    refused(opened, ctx, odd[..., :64], odd[..., :64], two_heads, two_heads, torch.bfloat16, match="multiple of 16")
    flat = dev(2 * 16 * 64 + 8)[8:].view(2, 16, 1, 64)
    refused(opened, ctx, flat, flat, e, e, torch.bfloat16, match="aligned")
    shifted = torch.zeros(33, dtype=torch.uint8, device="cuda")[1:].view(2, 1, 16)
    refused(opened, ctx, k, k, shifted, e, torch.bfloat16, match="k_exp is not")
    refused(opened, ctx, k, k, e, shifted, torch.bfloat16, match="v_exp is not")

    c = opened(ctx, k, k.clone(), e, e.clone(), torch.bfloat16)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    read = kvdro.kvdro_kv_read
    for a, match, kind in (((i(0, 3), i(5), i(1)[None], out[:, :, :32], out), "shape", ValueError), ((i(0), i(5), i(1)[None], out, out), "q_off", ValueError),
                           ((i(0, 3), i(5, 6), i(1)[None], out, out), "kv_len", ValueError), ((i(0, 3), i(5), i(1), out, out), "table", ValueError),
                           ((i(0, 3), i(5), i(1)[None], out.half(), out), "dtype", TypeError), ((i(0, 3), i(5), i(1)[None], out, out[:2]), "shape", ValueError)):
        with pytest.raises(kind, match=match):
            read(c, *a)
    with pytest.raises(TypeError, match="dtype"):
        kvdro.kvdro_kv_append(c, out.half(), out, i(0, 1, 2))
    wide = torch.zeros((3, 1, 72), dtype=torch.bfloat16, device="cuda")
    refused(read, c, i(0, 3), i(5), i(1)[None], wide[..., 4:68], out, match="aligned")
    read(c, i(0, 3), i(5), i(1)[None], out[:0], out[:0])  # no tokens: nothing to do
    kvdro.kvdro_sync(ctx)
