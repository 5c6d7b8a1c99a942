"""The kernel for chunks: scales of either sign, rows that fill their warps and rows that do not."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv_support import Case  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 8, 2), ("fp16", 64, 7, 1), ("bf16", 64, 32, 1)])
@pytest.mark.parametrize("opt", [{}, {"softcap": 30.0}, {"window": 77}], ids=["plain", "cap", "window"])
def test_a_negative_scale_is_that_of_negated_queries(ctx, dtype, D, Hq, Hkv, opt):
    """-s q and s (-q) are the same numbers: equal bit for bit, over many pieces that each bring their Q."""
    case = Case([(700, 3000), (33, 40), (129, 1000), (300, 300), (90, 5000)], dtype, D, Hq, Hkv, 16, seed=1)
    out, lse = case.run(ctx, scale=-0.2, **opt)
    case.q = -case.q
    want, wz = case.run(ctx, scale=0.2, **opt)
    assert torch.equal(out, want) and torch.equal(lse, wz)
    case.q = -case.q
    case.check(out, lse, scale=-0.2, **opt)
    for _ in range(3):
        again = case.run(ctx, scale=-0.2, **opt)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("group", [1, 5, 8])
@pytest.mark.parametrize("window", [0, 150])
def test_rows_that_do_not_fill_a_warp_and_infinities_that_some_see(ctx, dtype, D, group, window):
    """Lanes of a warp without a row beside lanes with one, each of which adds the infinities that it sees by itself."""
    lens = [(n, n + 300) for n in (17, 31, 33, 50, 95, 127, 129, 200)]
    case = Case(lens, dtype, D, 2 * group, 2, 16, seed=group)
    clean, cz = case.run(ctx, window=window)
    case.check(clean, cz, window=window)
    sees = []
    for b, (n, kv) in enumerate(lens):
        at = [kv - 1, kv - n // 2, kv - n]  # the last row's own, one in the middle, the first row's
        v = case.values[b].clone()
        for i, j in enumerate(at):
            v[j, :, 3 + 32 * (i % (D // 32))::D] = float("inf")
        case.set(b, case.keys[b], v)
        p, j = torch.arange(kv - n, kv), torch.tensor(at)
        sees.append((j[None] <= p[:, None]) & ((j[None] > p[:, None] - window) if window else True))
    sees = torch.cat(sees)  # [T][3]
    out, lse = case.run(ctx, window=window)
    want = clean.clone()
    for i in range(3):
        d = 3 + 32 * (i % (D // 32))
        want[:, :, d] = torch.where(sees[:, i].cuda()[:, None], float("inf"), want[:, :, d])
    assert torch.equal(out, want) and torch.equal(lse, cz)
    kvdro.kvdro_sync(ctx)
