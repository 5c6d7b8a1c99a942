"""Values out of range in device memory: what is left out, what is reported, and what is nobody's business."""

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


def reported(ctx):
    with pytest.raises(kvdro.KvdroError) as e:
        kvdro.kvdro_sync(ctx)
    assert e.value.status == kvdro.KVDRO_ERANGE
    kvdro.kvdro_sync(ctx)  # once


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("bad", [-1, 20, 2 ** 31 - 1])
def test_a_returned_page_that_is_none_is_reported_and_stays_none(ctx, bad):
    """Request 1 is done; one of its three entries holds no page number."""
    n, page = 20, 16
    table = torch.full((2, 6), -1, dtype=torch.int32, device="cuda")
    table[0, :2], table[1, :3] = ints(4, 5), ints(7, bad, 9)
    ring = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    ring[18:], ring[:13] = ints(0, 1), ints(2, 3, 6, *range(10, 20))
    pool, held = ints(18, 15), ints(2, 3)
    held_out, pool_out, q_off, kv_len, slot = ints(0, 0), ints(0, 0), ints(0, 0, 0), ints(0, 0), ints(0)
    kvdro.kvdro_kv_plan(ctx, page, ints(20, 40), ints(1, -1), held, table, ring, pool, held_out, pool_out, q_off, kv_len, slot)
    reported(ctx)
    assert pool_out.tolist() == [18, 18] and held_out.tolist() == [2, 0]
    assert ring[13:16].tolist() == [7, -1, 9]
    assert slot.tolist() == [5 * page + 4]
    # the next request gets it: reported again, its token there has no slot
    table, held = table.clone(), ints(2, 0)
    slot, pos = torch.full((260,), 99, dtype=torch.int32, device="cuda"), torch.full((260,), 99, dtype=torch.int32, device="cuda")
    table = torch.cat([table, torch.full((2, 11), -1, dtype=torch.int32, device="cuda")], 1)
    kvdro.kvdro_kv_plan(ctx, page, ints(21, 0), ints(0, 260), held, table, ring, pool_out.clone(), held_out, pool_out, q_off, kv_len, slot, pos)
    reported(ctx)
    assert held_out.tolist() == [2, 17] and pool_out.tolist() == [15, 1] and kv_len.tolist() == [21, 260]
    assert table[1].tolist() == [0, 1, 2, 3, 6, *range(10, 20), 7, -1]
    assert pos.tolist() == list(range(260))
    assert slot.tolist() == [page * p + i for p in (0, 1, 2, 3, 6, *range(10, 20), 7) for i in range(page)] + [-1] * 4


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("q", [1, 3, 40, 300])
def test_pages_that_no_row_sees_are_nobodys_business(ctx, q, page):
    """Behind a window a server may have given pages away: their entries are not looked at, however the blocks lie."""
    for kv, window in ((500, 100), (777, 33), (1000, 512)):
        case = Case([(q, kv), (1, 5)], "bf16", 128, 8, 2, page, seed=q)
        first = max(0, kv - q - window + 1)  # the first position that a row sees
        case.table[0, :first // page] = -1
        out, lse = case.run(ctx, window=window)
        kvdro.kvdro_sync(ctx)
        assert worst(case, out, lse, 0, window=window) <= 1
        if first // page < kv // page:  # one that rows do see
            case.table[0, first // page] = -1
            case.run(ctx, window=window)
            reported(ctx)


@pytest.mark.parametrize("lens", [[(1, 200), (1, 100)], [(3, 200), (1, 100)], [(150, 200), (30, 40)]], ids=["token", "tokens", "chunk"])
@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("fp16", 64, 32)])
@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_a_request_with_a_bad_page_gets_its_other_positions(ctx, lens, dtype, D, page, bad):
    case = Case(lens, dtype, D, 8, 2, page, seed=4)
    case.table[0, 2] = bad
    out, lse = case.run(ctx)
    reported(ctx)
    assert worst(case, out, lse, 0, hidden=range(2 * page, 3 * page)) <= 1
    assert worst(case, out, lse, 1) <= 1


@pytest.mark.parametrize("T,Hkv,D", [(1, 1, 64), (33, 8, 128)])
def test_a_slot_that_is_none_leaves_the_cache_as_it_is(ctx, T, Hkv, D):
    n, page = 6, 16
    k, v = (torch.randn((n, page, Hkv, D), device="cuda").bfloat16() for _ in range(2))
    new = torch.randn((2, T, Hkv, D), device="cuda").bfloat16()
    slot = np.random.default_rng(T).permutation(n * page)[:T].astype(np.int32)
    cache = kvdro.kvdro_kv_open(ctx, k, v)
    for bad in (n * page, 2 ** 31 - 1, -2):
        slot[T // 2] = bad
        want = k.clone(), v.clone()
        for t in range(T):
            if t != T // 2:
                for w, x in zip(want, new):
                    w[slot[t] // page, slot[t] % page] = x[t]
        kvdro.kvdro_kv_append(cache, new[0], new[1], torch.from_numpy(slot).cuda())
        reported(ctx)
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    kvdro.kvdro_kv_close(cache)
