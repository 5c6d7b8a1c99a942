"""What the softmax weights and the pieces of split rows keep of a result, against 64 bits with tight bounds."""

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
    case.set(0, k, v)
    case.q.zero_()
    case.q[..., 0] = 3.5
    case.lens, case.keys, case.values, case.T = case.lens * B, [k] * B, [v] * B, B * q
    case.table, case.kv_len, case.q = case.table.repeat(B, 1), case.kv_len.repeat(B), case.q.repeat(B, 1, 1)
    case.off = np.arange(B + 1) * q
    case.q_off = torch.from_numpy(case.off.astype(np.int32)).cuda()
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
