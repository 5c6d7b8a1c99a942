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
