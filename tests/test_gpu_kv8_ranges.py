"""Caches of 8 bits at the ends of their ranges: pages that are none, values and keys near the type's largest, scores so large that FP32 rounds them."""

import copy
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv8_support import F64, Case8, Shared  # noqa: E402
from tests.kv_support import UNIT  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


def spoil_page_zero(case, *tables):
    """Nobody holds page 0 (what it held moves to a page that nobody has), and nobody wrote it: NaN codes, scale bytes of 255."""
    free = set(range(case.codes[0].shape[0])) - set(case.table[case.table >= 0].tolist())
    if 0 not in free:
        to = min(free)
        for a in (*case.codes, *case.exps):
            a[to] = a[0]
        for t in (case.table, *tables):
            t[t == 0] = to
    for a, x in zip((*case.codes, *case.exps), (0x7f, 0x7f, 255, 255)):
        a[0] = x


def without(case, b, first, n):
    """The case as ``check`` takes it, positions first .. first + n - 1 of request b, which all of its rows would see, left out."""
    c = copy.copy(case)
    c.lens, c.keys, c.values = list(case.lens), list(case.keys), list(case.values)
    q, kv = c.lens[b]
    assert kv - q >= first + n
    c.lens[b] = (q, kv - n)
    for x in (c.keys, c.values):
        x[b] = torch.cat([x[b][:first], x[b][first + n:]])
    return c


def reported(ctx):
    with pytest.raises(kvdro.KvdroError) as e:
        kvdro.kvdro_sync(ctx)
    assert e.value.status == kvdro.KVDRO_ERANGE


@pytest.mark.parametrize("q", [1, 3, 6, 20, 300])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("fp16", 64, 32), ("bf16", 64, 128), ("fp16", 128, 64)])
@pytest.mark.parametrize("opt", [{}, {"softcap": 30.0}], ids=["plain", "cap"])
def test_a_page_that_is_none_is_left_out(ctx, q, dtype, D, page, opt):
    """In the middle of a request, where every row sees the whole block; nothing of any other page takes its place."""
    case = Case8([(q, 1500), (1, 100)], dtype, D, 8, 2, page, seed=q)
    spoil_page_zero(case)
    for bad in (-1, 10 ** 6):
        case.table[0, 2] = bad
        out, lse = case.run(ctx, **opt)
        reported(ctx)
        without(case, 0, 2 * page, page).check(out, lse, **opt)


@pytest.mark.parametrize("lens", [[(1, 100), (1, 30)], [(1, 100)] * 12, [(40, 90), (1, 30)]], ids=["few", "tokens", "chunk"])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("fp16", 64, 32)])
def test_a_page_of_a_prefix_that_is_none_is_left_out(ctx, lens, wide, dtype, D, page):
    s = Shared(lens, [0, len(lens)], [700], bits=8, wide=wide, dtype=dtype, D=D, Hq=8, Hkv=2, page=page, seed=2)
    spoil_page_zero(s.c, s.table, s.prefix_table)
    s.prefix_table[0, 3] = -1
    out, lse = s.run(ctx)
    reported(ctx)
    for x in (s.c.keys, s.c.values):
        x[s.B] = torch.cat([x[s.B][:3 * page], x[s.B][4 * page:]])
    s.check(out, lse)


def large_values(case, e):
    """The values of every request within 1.7 * 2^e, whatever is asked of the scale: 448 * 2^119 = 1.75 * 2^127."""
    g = torch.Generator(device="cuda").manual_seed(e + 200)
    for b, (_, kv) in enumerate(case.lens):
        v = (2 * torch.rand((kv, case.Hkv, case.D), generator=g, device="cuda", dtype=F64) - 1) * 1.7 * 2.0 ** e
        case.set(b, case.keys[b].to(case.dt), v.to(case.dt))


@pytest.mark.parametrize("q", [1, 3, 6])
@pytest.mark.parametrize("n", [1, 2, 40, 3000])
@pytest.mark.parametrize("e", [-118, 113, 121, 125, 127])
def test_few_rows_over_values_near_the_largest(ctx, q, n, e):
    """BF16: a mean of values is no larger than they are, however many, one request alone (pieces joined) or many; and the smallest."""
    for B, D in ((1, 128), (200, 64)):
        case = Case8([(q, n)] * B, "bf16", D, 8, 2, 16, seed=n)
        large_values(case, e)
        out, lse = case.run(ctx, causal=False)
        kvdro.kvdro_sync(ctx)
        case.check(out, lse, causal=False, only={0, B - 1})


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("e", [-118, 113, 121, 125, 127])
def test_prefixes_of_values_near_the_largest(ctx, wide, e):
    for n in (1, 3000):
        s = Shared([(1, 1), (1, 300), (2, 40)], [0, 3], [n], bits=8, wide=wide, dtype="bf16", D=128, Hq=8, Hkv=2, page=16, seed=3)
        large_values(s.c, e)
        out, lse = s.run(ctx)
        kvdro.kvdro_sync(ctx)
        s.check(out, lse)


@pytest.mark.parametrize("q,n,e", [(40, 1, 127), (300, 1, 121), (40, 3000, 106)])
def test_chunks_over_large_values(ctx, q, n, e):
    """Their sums are not divided before the end: n weights of up to 2^8 times values of up to 2^(e + 1) have to stay below 2^128."""
    case = Case8([(q, n)], "bf16", 128, 8, 2, 16, seed=n)
    large_values(case, e)
    out, lse = case.run(ctx, causal=False)
    kvdro.kvdro_sync(ctx)
    case.check(out, lse, causal=False)


@pytest.mark.parametrize("q", [1, 3, 6, 40])
@pytest.mark.parametrize("n", [1, 40, 700])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64), ("fp16", 128)])
def test_large_scores_leave_a_mean_a_mean(ctx, q, n, dtype, D):
    """All keys are the same one, so that the scores are equal whatever FP32 makes of them, and the result is the mean of the values, which
    differ in size.  Off by u for its own rounding, u for its weights' (FP16 ones of at least 2^-7: normal numbers) and 2^-18 for exponentials
    and sums: no part of a score."""
    case = Case8([(q, n)], dtype, D, 8, 2, 16, seed=n, spread=6.0)
    k = torch.zeros((n, 2, D), device="cuda", dtype=case.dt)
    k[..., 0] = 1.0
    case.set(0, k, case.values[0].to(case.dt))
    case.q.zero_()
    case.q[..., 0] = 1.3671875
    u, v = UNIT[case.dt], case.values[0].repeat_interleave(4, 1)
    ref, size = v.mean(0), v.abs().mean(0)
    tol = u * ref.abs() + (u + 2.0 ** -18) * size + (2.0 ** -25 if dtype == "fp16" else 0.0)
    for x in range(0, 27):
        # in units of log2 just below 2^x too, where a score and a value's exponent together may need a bit more
        for scale in (2.0 ** x, -2.0 ** x, 2.0 ** x * 0.9999 / 1.3671875 * math.log(2)):
            out, lse = case.run(ctx, causal=False, scale=scale)
            assert torch.isfinite(lse).all()
            worst = ((out.to(F64) - ref).abs() / tol).max()
            assert worst <= 1, (scale, float(worst))
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("q", [1, 3, 6, 40])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("B", [1, 300])
def test_scores_so_large_that_their_spacing_matters(ctx, q, dtype, D, B):
    """Scores of 2^16 to 2^27 that climb or fall in small steps, over values of sizes of 2^-6 to 2^6: whatever FP32 makes of them, a result is a
    mean of values."""
    kv = 2000
    case = Case8([(q, kv)], dtype, D, 4, 1, 16, seed=1, spread=6.0)
    v = case.values[0].to(case.dt)
    case.table, case.kv_len, case.q = case.table.repeat(B, 1), case.kv_len.repeat(B), case.q.repeat(B, 1, 1)
    case.lens, case.T = case.lens * B, B * q
    case.q_off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * q
    held = case.values[0].abs().amax(0).clamp(min=0) * 1.01
    codes = torch.arange(0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).float()
    climb = codes[torch.arange(kv, device="cuda") * 127 // kv]
    for e in range(16, 27):
        for step, keys in ((0.05, climb), (0.4, climb), (0.05, climb.flip(0))):
            k = torch.zeros((kv, 1, D), device="cuda")
            k[..., 0], k[..., 1] = 448.0, keys[:, None]
            case.set(0, k.to(case.dt), v)
            case.q.zero_()
            case.q[..., 0], case.q[..., 1] = 1.0, step * 2.0 ** (8 - e)
            for scale in (2.0 ** (e - 8), -2.0 ** (e - 8)):
                out, lse = case.run(ctx, scale=scale, max_q=q)
                assert torch.isfinite(lse).all() and torch.isfinite(out).all(), (e, step, scale)
                assert (out.to(F64).abs() <= held).all(), (e, step, scale)
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("q", [1, 3, 6, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_keys_near_the_largest_and_small_queries(ctx, q, D):
    """Scores of ordinary size from keys of 2^125 and queries of 2^-110, and from small keys and large queries; a query of zeros beside them."""
    for up, down in ((125, -110), (-120, 110)):
        case = Case8([(q, 300), (1, 40)], "bf16", D, 8, 2, 16, seed=q)
        for b in range(2):
            case.set(b, (case.keys[b].clamp(-3, 3) * 2.0 ** up).to(case.dt), case.values[b].to(case.dt))
        case.q = (case.q.to(F64).clamp(-3, 3) * 2.0 ** down).to(case.dt)
        case.q[0, ::3] = 0
        scale = 2.0 ** (-up - down - 3)
        out, lse = case.run(ctx, scale=scale)
        kvdro.kvdro_sync(ctx)
        case.check(out, lse, scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_beyond_fp16_in_attention(ctx, D):
    """A cache that was written as BF16 and is opened as FP16.  Few rows multiply codes, which are no larger than 448, whatever the scale: values
    and keys beyond FP16 count as they are.  Chunks widen them to FP16, as reads do: infinities."""
    for q in (1, 3, 6, 40):
        case = Case8([(q, 100), (1, 50)], "bf16", D, 8, 2, 16, seed=q)
        k, v = case.keys[0].to(case.dt), case.values[0].to(case.dt)
        v[5, :, 3] = 3.0e5  # every row sees it, at a weight of about 1 / 100: a result that FP16 holds
        case.set(0, k, v)
        case.dt, case.q = torch.float16, case.q.to(torch.float16) * 0.25
        out, lse = case.run(ctx)
        kvdro.kvdro_sync(ctx)
        if q < 40:
            case.check(out, lse)
        else:
            assert torch.isinf(out[:q, :, 3]).all() and torch.isfinite(out[:q, :, 4:]).all()
        k[5, :, 7], v[5, :, 3] = -2.0 ** 17, 1.0
        case.dt = torch.bfloat16
        case.set(0, k, v)
        case.dt = torch.float16
        case.q[..., 7] = 2.0 ** -14
        out, lse = case.run(ctx)
        kvdro.kvdro_sync(ctx)
        if q < 40:
            case.check(out, lse)
        else:  # a score of -infinity
            case.keys[0], case.values[0] = (torch.cat([x[0][:5], x[0][6:]]) for x in (case.keys, case.values))
            case.lens[0] = (q, 99)
            case.check(out, lse)
