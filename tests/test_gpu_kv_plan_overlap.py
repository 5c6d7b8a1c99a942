"""A plan whose results would overwrite what it reads is refused."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402

B, MAX_PAGES, PAGES, T = 6, 4, 40, 9
SIZES = {"cached": B, "new_len": B, "reserve": B, "held": B, "pool": 2, "table": B * MAX_PAGES, "ring": PAGES, "held_out": B, "pool_out": 2,
         "q_off": B + 1, "kv_len": B, "slot": T, "pos": T}
READ = ("cached", "new_len", "reserve", "held", "pool")


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


def arrays(store, at):
    a = {k: store[at[k]:at[k] + n] for k, n in SIZES.items()}
    a["table"] = a["table"].view(B, MAX_PAGES)
    return a


def side_by_side():
    at, end = {}, 0
    for k, n in SIZES.items():
        at[k], end = end, end + n
    return at, end


def fill(a):
    a["cached"].zero_()
    a["new_len"].fill_(1)
    a["held"].zero_()
    a["table"].fill_(-1)
    a["ring"].copy_(torch.arange(PAGES))
    a["pool"].copy_(torch.tensor([0, PAGES]))
    a["reserve"].zero_()


def test_arrays_side_by_side_are_fine(ctx):
    at, end = side_by_side()
    store = torch.full((end,), -9, dtype=torch.int32, device="cuda")
    a = arrays(store, at)
    fill(a)
    kvdro.kvdro_kv_plan(ctx, 16, **a)
    kvdro.kvdro_sync(ctx)
    assert a["kv_len"].tolist() == [1] * B and a["slot"].tolist() == [16 * b for b in range(B)] + [-1] * (T - B)


@pytest.mark.parametrize("written", [k for k in SIZES if k not in READ])
def test_results_over_anything_else_are_refused(ctx, written):
    at, end = side_by_side()
    for other in SIZES:
        if other == written:
            continue
        for shift in (0, SIZES[other] - 1, 1 - SIZES[written]):  # the same place, the last element, the first
            room = 64
            where = {k: x + room for k, x in at.items()}
            where[written] = where[other] + shift
            store = torch.full((end + 2 * room,), -9, dtype=torch.int32, device="cuda")
            a = arrays(store, where)
            fill(a)
            before = store.clone()
            with pytest.raises(kvdro.KvdroError, match="overlaps") as e:
                kvdro.kvdro_kv_plan(ctx, 16, **a)
            assert e.value.status == kvdro.KVDRO_EINVAL
            assert torch.equal(store, before), (written, other)
    kvdro.kvdro_sync(ctx)


@pytest.mark.parametrize("name", ["reserve", "held"])
def test_inputs_may_share(ctx, name):
    """What is only read may be the same array twice."""
    at, end = side_by_side()
    store = torch.zeros(end, dtype=torch.int32, device="cuda")
    a = arrays(store, at)
    fill(a)
    a[name] = a["cached"]
    kvdro.kvdro_kv_plan(ctx, 16, **a)
    kvdro.kvdro_sync(ctx)
    assert a["kv_len"].tolist() == [1] * B
