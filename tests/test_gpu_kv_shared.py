"""Attention of requests that share prefixes, on the GPU against 64 bits."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv8_support import Shared  # noqa: E402

# requests' (new tokens, tokens with them), bounds of the requests that share each prefix, and prefixes' lengths
ONE = ([(1, 30), (1, 1), (1, 200), (1, 77)], [0, 4], [333])
FEW = ([(1, 30), (1, 9)], [0, 2], [1000])
MANY = ([(1, 20 + 7 * i) for i in range(90)], [0, 90], [517])
GROUPS = ([(1, 5), (2, 40), (3, 0), (1, 100), (4, 2), (0, 12), (1, 17), (130, 200), (1, 1), (3, 64)], [1, 4, 4, 6, 9], [129, 50, 16, 1])
NONE = ([(1, 40), (5, 60), (1, 9)], [1, 2, 3], [0, 0])
CHUNKS = ([(300, 300), (40, 300), (1, 700)], [0, 2, 3], [600, 128])


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("case", [ONE, FEW, MANY, GROUPS, NONE, CHUNKS], ids=["one", "few", "many", "groups", "none", "chunks"])
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,layout", [("bf16", 128, 8, 2, 16, "dense"), ("fp16", 64, 14, 2, 32, "packed"),
                                                        ("bf16", 64, 4, 4, 128, "heads_first"), ("fp16", 128, 20, 1, 64, "dense")])
def test_prefixes_and_own_tokens(ctx, wide, bits, case, dtype, D, Hq, Hkv, page, layout):
    s = Shared(*case, bits=bits, wide=wide, dtype=dtype, D=D, Hq=Hq, Hkv=Hkv, page=page, layout=layout, seed=D + Hq)
    a, b = s.run(ctx), s.run(ctx)
    kvdro.kvdro_sync(ctx)
    s.check(*a)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])  # the order of sums is fixed


@pytest.mark.parametrize("opt", [dict(causal=False), dict(softcap=30.0), dict(softcap=0.5), dict(scale=0.3), dict(scale=-0.1), dict(scale=0.0)],
                         ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
def test_masks_caps_and_scales(ctx, wide, bits, opt):
    for case in (ONE, GROUPS, CHUNKS):
        if opt.get("causal") is False:  # whole() has no rows in front of position 0
            case = ([(min(q, kv), kv) for q, kv in case[0]], *case[1:])
        s = Shared(*case, bits=bits, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=11)
        s.check(*s.run(ctx, **opt), **opt)
        kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("bits", [16, 8])
def test_long_prefixes_are_split_and_joined(ctx, bits):
    for case, kw in ((([(1, 300), (1, 5000), (1, 20)] * 9, [0, 27], [40001]), dict(dtype="bf16", D=128, Hq=8, Hkv=2, page=64)),
                     (([(1, 9), (2, 70), (1, 4000)], [0, 1, 3], [20000, 33333]), dict(dtype="fp16", D=64, Hq=16, Hkv=4, page=16))):
        s = Shared(*case, bits=bits, seed=3, **kw)
        a, b = s.run(ctx), s.run(ctx)
        kvdro.kvdro_sync(ctx)
        s.check(*a)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("side", ["prefix", "own"])
def test_one_side_has_all_the_weight(ctx, bits, side):
    """Scores hundreds apart between the prefix and the request's own tokens."""
    for wide in (False, True):
        for q in (1, 50):
            s = Shared([(1, 100), (1, 40), (q, 60)], [0, 3], [300], bits=bits, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=5)
            for b in range(4):
                if (b == 3) == (side == "prefix"):
                    s.c.keys[b] = (s.c.keys[b] * 60).to(s.c.dt)
                    s.c.set(b, s.c.keys[b], s.c.values[b].to(s.c.dt))
            s.check(*s.run(ctx))
            kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("wide", [False, True])
def test_whatever_max_q_says(ctx, wide):
    for bits in (16, 8):
        s = Shared(*GROUPS, bits=bits, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=6)
        for max_q in (0, 1, 3, 130, 5000):
            s.check(*s.run(ctx, max_q=max_q))
            kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D,page", [(128, 16), (64, 128), (64, 32)])
def test_prefixes_that_end_anywhere(ctx, bits, D, page):
    """Around the ends of pages, slices and blocks, where each request reads its own; pages behind the end are none, and hold NaN."""
    lengths = [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 0]
    lens = [(1 + i % 2, 1 + 37 * i % 300) for i in range(2 * len(lengths) + 2)]
    s = Shared(lens, list(range(0, 2 * len(lengths) + 1, 2)), lengths, bits=bits, dtype="fp16", D=D, Hq=8, Hkv=2, page=page, seed=12)
    s.check(*s.run(ctx))
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("bits", [16, 8])
def test_values_of_nan_in_own_tokens_that_some_rows_see(ctx, bits):
    """A row that does not see them is as if they were not there, its prefix beside them."""
    make = lambda wide: Shared([(4, 200), (1, 9)], [0, 2], [77], bits=bits, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=13)  # noqa: E731
    for wide in (False, True):
        s, clean = make(wide), make(wide)
        v = s.c.values[0].to(s.c.dt)
        v[199, :, ::7] = float("nan")
        s.c.set(0, s.c.keys[0].to(s.c.dt), v)
        (out, lse), (want, wz) = s.run(ctx), clean.run(ctx)
        kvdro.kvdro_sync(ctx)
        assert torch.isnan(out[3][:, ::7]).all() and torch.isfinite(out[:3]).all() and torch.isfinite(out[4]).all()
        out[3], lse[3] = want[3], wz[3]
        clean.check(out, lse)


def test_nan_in_the_scratch_does_not_matter(ctx):
    for case in (GROUPS, NONE, ONE):
        s = Shared(*case, wide=True, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=7)
        work = torch.full((kvdro.kvdro_kv_shared_bytes(s.T, 8, 128) // 4,), float("nan"), dtype=torch.float32, device="cuda")
        s.check(*s.run(ctx, work=work))
        kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("wide", [False, True])
def test_bounds_out_of_range_are_reported(ctx, wide):
    i32 = dict(dtype=torch.int32, device="cuda")
    for share, lengths in (([0, 5, 3, 4], [300] * 3), ([-1, 2, 3, 4], [300] * 3), ([0, 1, 2, 9], [300] * 3), ([0, 1, 2, 4], [300, -7, 300]),
                           ([0, 1, 2, 4], [300, 10 ** 9, 300])):
        s = Shared(ONE[0], [0, 1, 2, 4], [300] * 3, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=6)
        s.share_off, s.prefix_len = torch.tensor(share, **i32), torch.tensor(lengths, **i32)
        s.run(ctx)
        with pytest.raises(kvdro.KvdroError) as e:
            kvdro.kvdro_sync(ctx)
        assert e.value.status == kvdro.KVDRO_ERANGE
    s = Shared(*ONE, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=6)
    s.prefix_table[0, 3] = -1
    out, _ = s.run(ctx)
    with pytest.raises(kvdro.KvdroError) as e:
        kvdro.kvdro_sync(ctx)
    assert e.value.status == kvdro.KVDRO_ERANGE and torch.isfinite(out).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("case,wide", [(GROUPS, True), (ONE, True), (ONE, False)], ids=["groups", "once", "each"])
def test_captured_and_replayed(ctx, bits, case, wide):
    """New queries and lengths in the same arrays; a workspace of its own for the graph."""
    s = Shared(*case, bits=bits, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=8)
    s.run(ctx)  # loads the kernels
    cache, work = s.open(ctx), torch.empty(kvdro.kvdro_kv_shared_bytes(s.T, 8, 128), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = s.run(ctx, work=work, cache=cache)
    for seed in (1, 2):
        s.c.q.copy_(torch.randn(s.c.q.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        s.check(out, lse)
    s.prefix_len[0] = 0
    graph.replay()
    torch.cuda.synchronize()
    want = s.run(ctx, cache=cache)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    kvdro.kvdro_sync(ctx)


def test_on_another_stream_and_without_scratch(ctx):
    s = Shared(*MANY, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=9)
    want = s.run(ctx)
    stream = torch.cuda.Stream()
    for _ in range(3):
        got = s.run(ctx, stream=stream)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    kvdro.kvdro_sync(ctx)


def test_tokens_behind_the_last_request(ctx):
    s = Shared(*ONE, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=10)
    s.c.q = torch.cat([s.c.q, s.c.q[:3]])
    s.T += 3
    out, lse = s.run(ctx)
    kvdro.kvdro_sync(ctx)
    assert (out[-3:] == 0).all() and (lse[-3:] == -float("inf")).all()
    s.check(out, lse)


def test_refusals(ctx):
    s = Shared(*ONE, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=10)
    need = kvdro.kvdro_kv_shared_bytes(s.T, 8, 128)
    assert need == s.T * 8 * 130 * 4
    store = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    for work, match in ((store[:need - 1], "work has"), (store[1:need + 1], "aligned")):
        with pytest.raises(kvdro.KvdroError, match=match) as e:
            s.run(ctx, work=work)
        assert e.value.status == kvdro.KVDRO_EINVAL
    with pytest.raises(ValueError, match="work"):
        s.run(ctx, work=torch.empty(need, dtype=torch.uint8))
    for opt, match in ((dict(scale=float("inf")), "scale"), (dict(softcap=-1.0), "softcap"), (dict(max_q=-1), "max_q")):
        with pytest.raises(kvdro.KvdroError, match=match):
            s.run(ctx, **opt)
    s.share_off = torch.zeros(6, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="share_off"):
        s.run(ctx)
    s.share_off, s.prefix_len = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    s.prefix_table = torch.zeros((5, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(kvdro.KvdroError, match="G = 5"):
        s.run(ctx)
    for T, heads, d in ((-1, 8, 128), (1, 0, 128), (1, 8, 96), (1 << 30, 4096, 64)):
        with pytest.raises(kvdro.KvdroError):
            kvdro.kvdro_kv_shared_bytes(T, heads, d)
