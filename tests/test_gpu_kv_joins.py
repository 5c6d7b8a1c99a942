"""Chunks whose tiles are split: every number of tiles at which their pieces are joined in another way, on the GPU against 64 bits."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv8_support import Case8, Shared  # noqa: E402
from tests.kv_support import Case  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


# One tile of 30 rows a request, each of which several CTAs share.  On 152 SMs up to 14 tiles have four CTAs for the columns (heads of 128), up to
# 28 two, up to 38 one; the host counts 30 B / 256 tiles more, so that 34 are the last and 35 the first on either side.
@pytest.mark.parametrize("B", [1, 14, 15, 28, 29, 34, 35, 60])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("fp16", 64, 64)])
def test_tiles_of_one_row_tile_each(ctx, B, bits, dtype, D, page):
    case = (Case8 if bits == 8 else Case)([(30, 1500 + 7 * b) for b in range(B)], dtype, D, 1, 1, page, seed=B)
    a, b = case.run(ctx), case.run(ctx)
    kvdro.kvdro_sync(ctx)
    case.check(*a)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])  # the order of sums is fixed


@pytest.mark.parametrize("G", [1, 14, 15, 28, 29, 34, 35])
@pytest.mark.parametrize("bits", [16, 8])
def test_prefixes_of_one_row_tile_each(ctx, G, bits):
    """Their sums are left for the requests' own launch."""
    lens = [(5, 20)] * (6 * G)
    s = Shared(lens, list(range(0, 6 * G + 1, 6)), [1500 + 7 * g for g in range(G)], bits=bits, wide=True, dtype="bf16", D=128, Hq=1, Hkv=1, page=16, seed=G)
    a, b = s.run(ctx), s.run(ctx)
    kvdro.kvdro_sync(ctx)
    s.check(*a)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
