"""The page plan and the append on the GPU, against plain restatements; what they leave out when values are out of range."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests import kv_support  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


def plan_inputs(seed, B, page, max_pages, n, new, p_new=0.3, p_done=0.1, fill=0.5, reserve=True, head=None):
    rng = np.random.default_rng(seed)
    cap = max_pages * page
    cached = np.minimum((rng.random(B) ** 2 * (fill * n * page / B)).astype(np.int64), cap)
    fresh = rng.random(B) < p_new
    new_len = np.where(fresh, 1 + (rng.random(B) * new).astype(np.int64), 1)
    new_len[rng.random(B) < p_done] = -1
    new_len[rng.random(B) < 0.05] = 0
    held = -(-cached // page)
    extra = rng.integers(0, 3, B)  # some hold more than their tokens fill
    held = np.minimum(np.where(held.sum() + extra.cumsum() <= n, held + extra, held), max_pages)
    owner = rng.permutation(n)
    table = np.full((B, max_pages), -1)
    table[np.arange(max_pages)[None] < held[:, None]] = owner[:held.sum()]
    free = owner[held.sum():]
    head = int(rng.integers(n)) if head is None else head
    ring = np.full(n, -1)
    ring[(head + np.arange(len(free))) % n] = free
    res = (rng.random(B) * 2 * cap * (rng.random(B) < 0.5)).astype(np.int64) if reserve else None
    return {"cached": cached, "new_len": new_len, "reserve": res, "held": held, "table": table, "ring": ring,
            "pool": np.array([head, len(free)]), "T": int(np.maximum(new_len, 0).sum()) + 5}


def run_plan(ctx, page, i, pos=True, times=1):
    d = {k: torch.from_numpy(np.ascontiguousarray(v, np.int32)).cuda() for k, v in i.items() if isinstance(v, np.ndarray)}
    B = len(i["cached"])
    o = {"held_out": B, "pool_out": 2, "q_off": B + 1, "kv_len": B, "slot": i["T"], "pos": i["T"]}
    o = {k: torch.full((n,), -99, dtype=torch.int32, device="cuda") for k, n in o.items()}
    for _ in range(times):
        kvdro.kvdro_kv_plan(ctx, page, d["cached"], d["new_len"], d["held"], d["table"], d["ring"], d["pool"], o["held_out"],
                            o["pool_out"], o["q_off"], o["kv_len"], o["slot"], o["pos"] if pos else None, reserve=d.get("reserve"))
    return {k: v.cpu().numpy() for k, v in {**d, **o}.items()}


@pytest.mark.parametrize("seed,B,page,max_pages,n,new,fill", [
    (1, 1, 16, 4, 8, 5, 0.5), (2, 7, 16, 9, 40, 60, 0.5), (3, 513, 32, 40, 3000, 300, 0.6), (4, 512, 16, 64, 20000, 900, 0.5),
    (5, 1000, 128, 16, 2500, 700, 0.8), (6, 4097, 16, 128, 90000, 1000, 0.4), (7, 16384, 64, 33, 70000, 40, 0.5),
    (8, 64, 16, 8, 100, 100, 0.9)])
def test_plan(ctx, seed, B, page, max_pages, n, new, fill):
    for reserve in (True, False):
        i = plan_inputs(seed, B, page, max_pages, n, new, fill=fill, reserve=reserve)
        want = kv_support.plan(page, i)
        got = run_plan(ctx, page, i, times=2)  # a second call gives the same
        for k, v in want.items():
            assert np.array_equal(got[k], v), k
    kvdro.kvdro_sync(ctx)


def test_plan_runs_a_server_until_every_page_is_back(ctx):
    """Requests come, grow, are refused when pages run out, and leave; the pages in tables and ring stay a partition."""
    rng = np.random.default_rng(3)
    B, page, mp, n = 20, 16, 12, 97
    i = {"cached": np.zeros(B, np.int64), "held": np.zeros(B, np.int64), "table": np.full((B, mp), -1), "ring": rng.permutation(n),
         "pool": np.array([90, n]), "reserve": np.zeros(B, np.int64)}
    running, refused = np.zeros(B, bool), 0
    for step in range(60):
        last = step >= 50
        new = np.zeros(B, np.int64)
        for b in range(B):
            if running[b]:
                new[b] = -1 if last or rng.random() < 0.08 else 1
            elif not last and rng.random() < 0.5:
                new[b] = rng.integers(1, 60)
                i["reserve"][b] = new[b] + rng.integers(0, 100)
        i |= {"new_len": new, "T": int(np.maximum(new, 0).sum())}
        want = kv_support.plan(page, i)
        got = run_plan(ctx, page, i, pos=step % 2 == 0)
        for k in want:
            if k != "pos" or step % 2 == 0:
                assert np.array_equal(got[k], want[k]), (step, k)
        done, ok = new < 0, (got["kv_len"] > 0) & (new > 0)
        refused += int(((new > 0) & ~ok).sum())
        running = (running | ok) & ~done
        i["cached"] = np.where(done, 0, np.where(ok, got["kv_len"], i["cached"]))
        i |= {"held": got["held_out"], "table": got["table"], "ring": got["ring"], "pool": got["pool_out"]}
        head, free = got["pool_out"]
        mine = [int(p) for b in range(B) for p in got["table"][b, :got["held_out"][b]]]
        assert sorted(mine + [int(got["ring"][(head + x) % n]) for x in range(free)]) == list(range(n)), step
    assert refused and not running.any() and got["pool_out"][1] == n
    kvdro.kvdro_sync(ctx)


def test_plan_leaves_out_what_is_out_of_range(ctx):
    def bad(change, T=None):
        i = plan_inputs(11, 9, 16, 10, 60, 20, p_done=0.2)
        i["T"] = i["T"] if T is None else T
        change(i)
        got = run_plan(ctx, 16, i)
        with pytest.raises(kvdro.KvdroError) as e:
            kvdro.kvdro_sync(ctx)
        assert e.value.status == kvdro.KVDRO_ERANGE
        kvdro.kvdro_sync(ctx)  # reported once
        return i, got

    def put(name, at, v):
        return lambda i: i[name].__setitem__(at, v)
    for head, n in ((-1, 5), (60, 5), (0, 61), (3, -2)):
        i, got = bad(lambda i: i.__setitem__("pool", np.array([head, n])))
        assert np.array_equal(got["pool_out"], [head, n]) and np.array_equal(got["ring"], i["ring"])
        assert np.array_equal(got["table"], i["table"])
    for name, v in (("held", -1), ("held", 11), ("cached", -5), ("cached", 10 ** 6)):
        i, got = bad(put(name, 4, v))
        assert got["kv_len"][4] == 0
        at = slice(got["q_off"][4], got["q_off"][5])
        assert (got["slot"][at] == -1).all() and (got["pos"][at] == -1).all()
    # a page number in the ring that is none: the token that would get it has no slot
    i, got = bad(lambda i: i["ring"].__setitem__(slice(None), 60))
    fresh = got["held_out"] > i["held"]
    assert fresh.any() and all((got["table"][b, i["held"][b]:got["held_out"][b]] == -1).all() for b in np.nonzero(fresh)[0])
    i, got = bad(lambda i: None, T=1)  # more tokens than slots
    assert len(got["slot"]) == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,Hkv,D,page,layout", [(1, 1, 64, 16, "dense"), (3, 8, 128, 16, "packed"), (257, 3, 64, 32, "strided"),
                                                 (1000, 2, 128, 128, "heads_first"), (70, 40, 128, 64, "dense")])
def test_append(ctx, dtype, T, Hkv, D, page, layout):
    dt, rng = kv_support.DTYPES[dtype], np.random.default_rng(T)
    n = T // page + 3
    if layout == "heads_first":
        k, v = (torch.randn((n, Hkv, page, D), device="cuda").to(dt).transpose(1, 2) for _ in range(2))
    else:
        k, v = (torch.randn((n, page, Hkv, D), device="cuda").to(dt) for _ in range(2))
    qkv = torch.randn((T, 3 * Hkv, D), device="cuda").to(dt)
    k_new, v_new = qkv[:, Hkv:2 * Hkv], qkv[:, 2 * Hkv:]
    if layout == "strided":  # heads in reverse memory order are not allowed; rows with a gap are
        v_new = torch.randn((T, Hkv, D + 8), device="cuda").to(dt)[..., :D]
    if layout == "dense":
        k_new, v_new = k_new.contiguous(), v_new.contiguous()
    slot = rng.permutation(n * page)[:T].astype(np.int32)
    slot[rng.random(T) < 0.1] = -1
    want = [x.clone() for x in (k, v)]
    for t in np.nonzero(slot >= 0)[0]:
        want[0][slot[t] // page, slot[t] % page] = k_new[t]
        want[1][slot[t] // page, slot[t] % page] = v_new[t]
    cache = kvdro.kvdro_kv_open(ctx, k, v)
    kvdro.kvdro_kv_append(cache, k_new, v_new, torch.from_numpy(slot).cuda())
    kvdro.kvdro_sync(ctx)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    # a slot that is none is left out and reported
    slot[T // 2] = n * page
    kvdro.kvdro_kv_append(cache, k_new, v_new, torch.from_numpy(slot).cuda())
    with pytest.raises(kvdro.KvdroError) as e:
        kvdro.kvdro_sync(ctx)
    assert e.value.status == kvdro.KVDRO_ERANGE
    assert torch.equal(k, want[0]) or slot[T // 2] >= 0
    kvdro.kvdro_kv_close(cache)


def test_append_passes_32_bits_of_elements(ctx):
    """Pages 2^28 elements apart: the last lies past 2^32 elements."""
    n, page, Hkv, D = 18, 16, 1, 64
    store = torch.empty((n - 1) * (1 << 28) + 2 * page * D, dtype=torch.bfloat16, device="cuda")
    k = store.as_strided((n, page, Hkv, D), (1 << 28, D, D, 1))
    v = store.as_strided((n, page, Hkv, D), (1 << 28, D, D, 1), page * D)
    new = torch.randn((2, 3, 1, D), device="cuda").to(torch.bfloat16)
    slot = torch.tensor([17 * page + 5, 0, 16 * page + 15], dtype=torch.int32, device="cuda")
    cache = kvdro.kvdro_kv_open(ctx, k, v)
    kvdro.kvdro_kv_append(cache, new[0], new[1], slot)
    kvdro.kvdro_sync(ctx)
    for c, x in ((k, new[0]), (v, new[1])):
        assert torch.equal(c[17, 5], x[0]) and torch.equal(c[0, 0], x[1]) and torch.equal(c[16, 15], x[2])
    kvdro.kvdro_kv_close(cache)
