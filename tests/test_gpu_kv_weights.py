"""What the softmax weights, the cap and the pieces of split rows keep of a result, against 64 bits with tight bounds."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv_exact import worst  # noqa: E402
from tests.kv_support import Case  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


def repeat(case, B):
    """The one request of ``case`` B times, over the same pages."""
    q = case.lens[0][0]
    case.lens, case.keys, case.values, case.T = case.lens * B, case.keys * B, case.values * B, B * q
    case.table, case.kv_len, case.q = case.table.repeat(B, 1), case.kv_len.repeat(B), case.q.repeat(B, 1, 1)
    case.off = np.arange(B + 1) * q
    case.q_off = torch.from_numpy(case.off.astype(np.int32)).cuda()


@pytest.mark.parametrize("q", [1, 40])
@pytest.mark.parametrize("first", [0, 30000])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_many_small_weights_are_not_lost(ctx, q, first, dtype):
    """One key 17.5 above 32767 others, which alone carry a component: e^-17.5 is 2^-25.2, but 32767 of them make 8e-4."""
    case = Case([(q, 32768)], dtype, 128, 2, 1, 64, seed=1)
    k, v = torch.zeros_like(case.keys[0]), torch.zeros_like(case.values[0])
    k[first, :, 0] = 5.0
    v[:, :, 1], v[first, :, 1], v[first, :, 2] = 1.0, 0.0, 1.0
    case.keys[0], case.values[0] = k, v
    case.set(0, k, v)
    case.q.zero_()
    case.q[..., 0] = 3.5
    out, lse = case.run(ctx, scale=1.0)
    assert worst(case, out, lse, 0, scale=1.0) <= 1


@pytest.mark.parametrize("q", [1, 6, 40])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_many_small_weights_are_not_lost_where_one_cta_has_the_row(ctx, q, dtype):
    """The same with so many requests (over the same pages) that rows are not split: all small weights of a warp, or of the
    whole row, meet the large one."""
    B, kv = 600, 4096
    case = Case([(q, kv)], dtype, 128, 2, 1, 64, seed=1)
    k, v = torch.zeros_like(case.keys[0]), torch.zeros_like(case.values[0])
    k[0, :, 0] = 5.0
    v[:, :, 1], v[0, :, 1], v[0, :, 2] = 1.0, 0.0, 1.0
    case.keys[0], case.values[0] = k, v
    case.set(0, k, v)
    case.q.zero_()
    case.q[..., 0] = 3.5
    repeat(case, B)
    out, lse = case.run(ctx, scale=1.0)
    for b in (0, 1, 299, 599):
        assert worst(case, out, lse, b, scale=1.0) <= 1


@pytest.mark.parametrize("lens", [[(1, 20011)], [(2, 30000), (1, 5), (1, 9000)], [(300, 9001)], [(513, 513), (100, 5000), (1, 1)]],
                         ids=["token", "tokens", "chunk", "mixed"])
@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 8, 2, 16), (64, 16, 4, 64)])
def test_split_rows_within_bounds_of_their_weights(ctx, lens, D, Hq, Hkv, page):
    case = Case(lens, "fp16", D, Hq, Hkv, page, seed=9)
    out, lse = case.run(ctx)
    for b in range(len(lens)):
        assert worst(case, out, lse, b) <= 1
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("q", [1, 40])
@pytest.mark.parametrize("dtype,D", [("fp16", 64), ("fp16", 128), ("bf16", 128)])
@pytest.mark.parametrize("lead", [1.0, 1.25, 1.5, 1.75, -1.0, -1.5])
def test_scores_so_large_that_their_spacing_matters(ctx, q, dtype, D, lead):
    """Scores of 2^16 to 2^27 that climb in small steps: FP32 rounds them to multiples of up to 8, so that a row's maximum can
    pass the one its weights refer to by more than it seems.  Whatever the rounding, a result is a mean of values."""
    B, kv = 600, 2000  # so many that a row is not split
    case = Case([(q, kv)], dtype, D, 4, 1, 16, seed=1)
    k, v = torch.zeros_like(case.keys[0]), case.values[0]
    case.q.zero_()
    repeat(case, B)
    lo, hi = v.float().amin(0) - 0.01 * v.abs().max(), v.float().amax(0) + 0.01 * v.abs().max()
    for e in range(16, 27):
        for step in (0.02, 0.05, 0.011):
            k[..., 0], k[..., 1] = lead * 2.0 ** (e // 2), (torch.arange(kv, device="cuda") * step).to(case.dt)[:, None]
            case.set(0, k, v)
            case.q[..., 0], case.q[..., 1] = 2.0 ** (e - e // 2), 1.0
            out, lse = case.run(ctx, scale=1.0)
            assert torch.isfinite(lse).all() and torch.isfinite(out).all(), (e, step)
            assert ((out >= lo) & (out <= hi)).all(), (e, step)
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("cap", [0.5, 30.0, 50.0, 1000.0])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("n", [1, 300])
def test_a_capped_score_is_off_by_2_20_of_the_cap_at_most(ctx, cap, dtype, D, n):
    """With one visible key the log sum is the capped score.  Queries and keys of one component, so that the product
    is exact; scaling adds 2^-22 of the score, the units of log2 and back 2^-22 of the result."""
    B = 300 // n
    case = Case([(n, 1)] * B, dtype, D, 4, 1, 16, seed=1)
    for b in range(B):
        case.keys[b].zero_()
        case.keys[b][..., 0] = 1.0
        case.set(b, case.keys[b], case.values[b])
    case.q.zero_()
    x = torch.cat([torch.linspace(-5, 5, 600), torch.logspace(-6, 0, 300), -torch.logspace(-6, 0, 300)]).view(300, 4) * cap
    case.q[..., 0] = x.to(case.dt).cuda()
    out, lse = case.run(ctx, scale=1.0, softcap=cap, causal=False)
    x = case.q[..., 0].double()
    z = cap * torch.tanh(x / cap)
    tol = 2.0 ** -20 * cap + 2.0 ** -22 * (x.abs() / torch.cosh(x / cap) ** 2 + z.abs())
    assert ((lse.double() - z).abs() <= tol).all(), float(((lse.double() - z).abs() / tol).max())
    want = torch.cat([case.values[b] for b in range(B)]).repeat_interleave(n, 0).expand(-1, 4, -1)
    assert torch.equal(out, want)
