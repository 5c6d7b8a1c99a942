"""Caches of 8 bits on the GPU: rows quantised as they are written, read back, and attended to, against 64 bits."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv8_support import E4M3, F64, Case8, arrays, quantise, two  # noqa: E402
from tests.kv_support import DTYPES, Case  # noqa: E402

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


def rows_of_every_kind(dt, T, heads, D, seed):
    """Rows of many sizes: zeros, the type's smallest and largest, ties, sizes at the border of two scales, NaN and infinities."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((T, heads, D), generator=g, device="cuda").to(F64)
    lo, hi = (-130, 125) if dt == torch.bfloat16 else (-20, 13)
    x = x * two(torch.randint(lo, hi, (T, heads, 1), generator=g, device="cuda"))
    x = x.to(dt)
    big = torch.finfo(dt).max
    special = [torch.zeros(D), torch.full((D,), big), torch.full((D,), -big), torch.full((D,), torch.finfo(dt).tiny / 16),
               torch.cat([torch.tensor([448.0]), torch.arange(1, D) / 16]), torch.cat([torch.tensor([450.0]), torch.arange(1, D) / 16]),
               torch.cat([torch.tensor([float("nan"), float("inf"), -float("inf")]), torch.arange(3, D) / 8]), torch.full((D,), float("nan")),
               torch.cat([torch.tensor([1.0]), torch.full((D - 1,), 2.0 ** -12)])]
    for i, row in enumerate(special):
        x[i % T, i % heads] = row.to(dt).cuda()
    return x


@pytest.mark.parametrize("dtype,D,heads,page,layout,T", [("bf16", 128, 8, 16, "dense", 1), ("bf16", 128, 8, 16, "dense", 300), ("fp16", 64, 3, 32, "packed", 77),
                                                         ("bf16", 64, 1, 64, "heads_first", 40), ("fp16", 128, 5, 128, "dense", 129)])
def test_rows_are_quantised_as_they_are_written(ctx, dtype, D, heads, page, layout, T):
    dt, n = DTYPES[dtype], T // page + 9
    k, v = arrays(n, page, heads, D, layout, fill=0x11)
    exps = [torch.full((n, heads, page), 99, dtype=torch.uint8, device="cuda") for _ in "kv"]
    cache = kvdro.kvdro_kv_open8(ctx, k.view(E4M3), v.view(E4M3), *exps, dt)
    slot = torch.from_numpy(np.random.default_rng(T).permutation(n * page)[:T].astype(np.int32)).cuda()
    if T > 4:
        slot[2] = -1
    new = [rows_of_every_kind(dt, T, heads, D, T + i) for i in range(2)]
    packed = torch.cat(new, 1)
    kvdro.kvdro_kv_append(cache, packed[:, :heads], packed[:, heads:], slot)
    kvdro.kvdro_sync(ctx)
    keep = slot >= 0
    at = slot[keep].long()
    for rows, codes, e in zip(new, (k, v), exps):
        want, we = quantise(rows[keep])
        got = codes.reshape(-1, heads, D)[at].view(E4M3).to(F64)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
        assert torch.equal(e.transpose(1, 2).reshape(-1, heads)[at].long(), we + 127)
        # within half a step of e4m3, or of its smallest number
        x = rows[keep].to(F64)
        near = (got * two(we)[..., None] - x).abs() <= torch.maximum(x.abs() * 2.0 ** -4, two(we - 10)[..., None])
        assert (near | ~torch.isfinite(x)).all()
        rest = torch.ones(n * page, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert (codes.reshape(-1, heads, D)[rest] == 0x11).all() and (e.transpose(1, 2).reshape(-1, heads)[rest] == 99).all()


def gather(case, which, b, first, n):
    return (case.keys, case.values)[which][b][first:first + n].to(F64)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("dtype,D,Hkv,page,layout", [("bf16", 128, 8, 16, "dense"), ("fp16", 64, 3, 32, "packed"), ("bf16", 64, 1, 128, "heads_first")])
def test_rows_are_read_back(ctx, bits, dtype, D, Hkv, page, layout):
    """The last tokens of requests, some of none, some more than there are; strided results; what follows is left as it was."""
    lens = [(0, 40), (3, 3), (7, 200), (5, 0), (4, 2), (129, 129), (1, 1000)]
    case = (Case8 if bits == 8 else Case)(lens, dtype, D, Hkv, Hkv, page, seed=4, layout=layout)
    cache = case.open(ctx) if bits == 8 else kvdro.kvdro_kv_open(ctx, case.k, case.v)
    T = case.T + 3  # three tokens of no request
    store = torch.full((T + 2, 2 * Hkv, D), 5.0, dtype=case.dt, device="cuda")
    kvdro.kvdro_kv_read(cache, case.q_off, case.kv_len, case.table, store[:T, :Hkv], store[:T, Hkv:])
    kvdro.kvdro_sync(ctx)
    for which, got in enumerate((store[:T, :Hkv], store[:T, Hkv:])):
        want = torch.zeros((T, Hkv, D), dtype=F64, device="cuda")
        for b, (n, kv) in enumerate(lens):
            have = min(n, kv)
            if have:
                want[case.off[b + 1] - have:case.off[b + 1]] = gather(case, which, b, kv - have, have)
        assert torch.equal(got, want.to(case.dt))
    assert (store[T:] == 5).all()


def test_a_step_reads_what_it_wrote(ctx):
    """Slots and tables of one step: the read gives the rows as they were rounded."""
    n, page, heads, D, i32 = 40, 16, 2, 64, dict(dtype=torch.int32, device="cuda")
    k, v = arrays(n, page, heads, D, "dense")
    exps = [torch.zeros((n, heads, page), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in "kv"]
    cache = kvdro.kvdro_kv_open8(ctx, k.view(E4M3), v.view(E4M3), *exps, torch.bfloat16)
    table, ring, pool = torch.full((2, 20), -1, **i32), torch.randperm(n, device="cuda").to(torch.int32), torch.tensor([0, n], **i32)
    zero = torch.zeros(2, **i32)
    held, pool_out, q_off, kv_len, slot = torch.empty(2, **i32), torch.empty(2, **i32), torch.empty(3, **i32), torch.empty(2, **i32), torch.empty(101, **i32)
    kvdro.kvdro_kv_plan(ctx, page, zero, torch.tensor([1, 100], **i32), zero.clone(), table, ring, pool, held, pool_out, q_off, kv_len, slot)
    new = torch.randn((101, 2 * heads, D), device="cuda").bfloat16()
    kvdro.kvdro_kv_append(cache, new[:, :heads], new[:, heads:], slot)
    got = torch.empty((101, 2 * heads, D), dtype=torch.bfloat16, device="cuda")
    kvdro.kvdro_kv_read(cache, q_off, kv_len, table, got[:, :heads], got[:, heads:])
    kvdro.kvdro_sync(ctx)
    c, e = quantise(new)
    assert torch.equal(got.to(F64), c * two(e)[..., None])


def test_values_out_of_range_are_reported(ctx):
    case = Case8([(1, 100), (2, 40)], "bf16", 64, 4, 2, 16, seed=1)
    cache = case.open(ctx)
    k, v = (torch.full((3, 2, 64), 9.0, dtype=case.dt, device="cuda") for _ in "kv")
    table = case.table.clone()
    table[0, 6] = 10 ** 6
    for a in ((case.kv_len, table), (torch.tensor([100, -5], dtype=torch.int32, device="cuda"), case.table),
              (torch.tensor([100, 10 ** 6], dtype=torch.int32, device="cuda"), case.table)):
        kvdro.kvdro_kv_read(cache, case.q_off, *a, k, v)
        with pytest.raises(kvdro.KvdroError) as e:
            kvdro.kvdro_sync(ctx)
        assert e.value.status == kvdro.KVDRO_ERANGE
        bad = slice(0, 1) if a[1] is table else slice(1, 3)
        assert (k[bad] == 0).all() and (v[bad] == 0).all()
        good = slice(1, 3) if a[1] is table else slice(0, 1)
        assert (k[good] != 0).any()
    kvdro.kvdro_kv_append(cache, k, v, torch.tensor([0, 10 ** 8, -2], dtype=torch.int32, device="cuda"))
    with pytest.raises(kvdro.KvdroError) as e:
        kvdro.kvdro_sync(ctx)
    assert e.value.status == kvdro.KVDRO_ERANGE


@pytest.mark.parametrize("lens", [MIX, DECODE], ids=["mix", "decode"])
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,layout", [
    ("bf16", 128, 8, 2, 16, "dense"), ("fp16", 64, 8, 8, 32, "packed"), ("bf16", 64, 14, 2, 64, "heads_first"),
    ("fp16", 128, 5, 1, 128, "heads_first"), ("bf16", 128, 16, 1, 16, "packed"), ("fp16", 128, 40, 1, 32, "dense"),
    ("bf16", 64, 3, 3, 16, "dense"), ("bf16", 128, 12, 2, 64, "dense"), ("fp16", 64, 8, 4, 128, "packed"),
    ("bf16", 64, 32, 1, 128, "dense")])
def test_types_heads_and_layouts(ctx, lens, dtype, D, Hq, Hkv, page, layout):
    check(ctx, Case8(lens, dtype, D, Hq, Hkv, page, seed=D + Hq, layout=layout))


@pytest.mark.parametrize("lens", [MIX, DECODE], ids=["mix", "decode"])
@pytest.mark.parametrize("opt", [dict(causal=False), dict(window=1), dict(window=7), dict(window=130), dict(softcap=5.0),
                                 dict(softcap=30.0, window=64), dict(softcap=0.01), dict(scale=0.5), dict(scale=-0.1), dict(scale=0.0)],
                         ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
def test_masks_caps_and_scales(ctx, lens, opt):
    check(ctx, Case8(lens, "bf16", 64, 8, 2, 16, seed=5), **opt)
    check(ctx, Case8(lens, "fp16", 128, 6, 3, 32, seed=6), **opt)


@pytest.mark.parametrize("lens", [[(1, 20011)], [(2, 30000), (1, 5), (1, 9000)], [(300, 9001)], [(1, 4096)] * 3, [(2000, 2000)],
                                  [(513, 513), (100, 5000), (1, 1), (17, 40)], [(1, 300)] * 200, [(9, 200)] * 33],
                         ids=lambda x: "_".join(f"{q}of{kv}" for q, kv in x[:3]) + f"x{len(x)}")
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", [("bf16", 128, 8, 2, 16), ("fp16", 64, 16, 4, 64), ("bf16", 128, 7, 1, 128)])
def test_lengths_that_are_split_and_joined(ctx, lens, dtype, D, Hq, Hkv, page):
    case = Case8(lens, dtype, D, Hq, Hkv, page, seed=9)
    check(ctx, case)
    a, b = case.run(ctx), case.run(ctx)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])  # the order of sums is fixed


@pytest.mark.parametrize("scores", [6.0, 40.0])
@pytest.mark.parametrize("lens", [[(1, 3000), (1, 77)], [(200, 1500), (3, 900)]], ids=["decode", "chunk"])
def test_scores_far_apart(ctx, lens, scores):
    """Running maxima that grow by hundreds on the way."""
    for dtype, D in (("bf16", 128), ("fp16", 64)):
        case = Case8(lens, dtype, D, 8, 2, 16, seed=3, scores=scores)
        for b, (_, kv) in enumerate(lens):  # ascending towards the end
            case.set(b, (case.keys[b] * torch.linspace(0.1, 1, kv, device="cuda")[:, None, None]).to(case.dt), case.values[b].to(case.dt))
        check(ctx, case)


@pytest.mark.parametrize("q", [1, 3, 40, 300])
@pytest.mark.parametrize("dtype,spread", [("bf16", 60.0), ("fp16", 9.0)])
def test_tokens_of_very_different_sizes(ctx, q, dtype, spread):
    """Values of 2^-60 beside ones of 2^60: the bound is of sum w |v|, which the largest dominate, and the smallest alone are tested by a
    request that holds no others."""
    case = Case8([(q, 900), (1, 300)], dtype, 128, 8, 2, 16, seed=q, spread=spread)
    small = (torch.randn((300, 2, 128), device="cuda") * 2.0 ** -spread).to(case.dt)
    case.set(1, case.keys[1].to(case.dt), small)
    check(ctx, case)


@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("fp16", 64, 64), ("fp16", 128, 32), ("bf16", 64, 16)])
@pytest.mark.parametrize("where", ["future", "window"])
@pytest.mark.parametrize("q", [1, 2, 5, 40, 300])
def test_what_a_row_does_not_see_does_not_matter(ctx, where, q, dtype, D, page):
    """Keys and values of NaN at a position that some rows of a request see and others do not."""
    kv, opt = 700, dict(window=200) if where == "window" else {}
    make = lambda: Case8([(q, kv), (1, 90)], dtype, D, 8, 2, page, seed=q)  # noqa: E731
    case, clean = make(), make()
    k, v = case.keys[0].to(case.dt), case.values[0].to(case.dt)
    at = kv - 1 if where == "future" else kv - q - 199 - 1 + (1 if q > 1 else 0)
    v[at, :, ::7] = float("nan")
    case.set(0, k, v)
    out, lse = case.run(ctx, **opt)
    kvdro.kvdro_sync(ctx)
    p = np.arange(kv - q, kv)
    sees = torch.from_numpy(np.concatenate([(p >= at) & ((p - at) < 200 if where == "window" else True), [False]])).cuda()
    want, wz = clean.run(ctx, **opt)
    assert torch.isfinite(out[~sees]).all()
    clean.check(torch.where(sees[:, None, None], want, out), torch.where(sees[:, None], wz, lse), **opt)
    assert torch.isnan(out[sees][..., ::7]).all()
    rest = torch.ones(D, dtype=torch.bool)
    rest[::7] = False
    assert torch.isfinite(out[sees][..., rest]).all()


def test_queries_of_every_size(ctx):
    """BF16 queries from 2^-110 to 2^100, a row of zeros, and infinities and NaN, whose rows alone they spoil."""
    for q in (1, 60):
        case = Case8([(q, 300)] * 8, "bf16", 128, 4, 2, 16, seed=8)
        for b, e in enumerate((-110, -30, 0, 3, 30, 60, 0, 0)):
            case.q[case.off[b]:case.off[b + 1]] *= 2.0 ** e
        case.q[case.off[2]:case.off[3]] = 0
        case.q[case.off[6], 1, 5] = float("nan")
        case.q[case.off[7], 2, 9] = float("inf")
        for b, e in ((4, -30), (5, -60)):  # scores of ordinary size
            case.set(b, (case.keys[b] * 2.0 ** e).to(case.dt), case.values[b].to(case.dt))
        out, lse = case.run(ctx)
        kvdro.kvdro_sync(ctx)
        case.check(out, lse, only=range(6))
        rows = torch.zeros((case.T, 4), dtype=torch.bool, device="cuda")
        rows[case.off[6], 1] = rows[case.off[7], 2] = True
        assert torch.isnan(out[rows]).all() and torch.isfinite(out[~rows]).all()


def test_fp16_keys_that_are_nearly_the_largest(ctx):
    """61440 and -61440 are what FP16's largest numbers become; scores stay finite."""
    for q in (1, 40):
        case = Case8([(q, 200)], "fp16", 64, 4, 2, 16, seed=2)
        v = case.values[0].to(case.dt)
        v[::3, :, ::5] = 65504.0
        v[1::3, :, ::5] = -65504.0
        case.set(0, case.keys[0].to(case.dt), v)
        assert float(case.values[0].abs().max()) == 61440.0
        check(ctx, case)
