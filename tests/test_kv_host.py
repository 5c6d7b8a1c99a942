"""Arguments that the page cache's binding refuses before it calls the library, and what the library refuses without a context."""

import ctypes

import pytest

from paper_2607_16892_gb300 import kvdro

torch = pytest.importorskip("torch")


def test_null_handles_are_refused():
    lib = kvdro.load_library()
    assert lib.kvdro_kv_close(None) == kvdro.KVDRO_OK
    assert lib.kvdro_kv_append(None, 1, None, None, None, None, None, None) == kvdro.KVDRO_EINVAL
    assert lib.kvdro_kv_attend(None, 1, 1, 1, 1, None, None, None, None, None, 1, 1.0, 1, 0, 0.0, None, None, None, None) == kvdro.KVDRO_EINVAL
    assert lib.kvdro_kv_plan(None, 16, 1, 1, 1, 1, *[None] * 14) == kvdro.KVDRO_EINVAL
    h = ctypes.c_void_p(5)
    assert lib.kvdro_kv_open(None, ctypes.byref(h), 0, 1, 16, 1, 64, None, None, None, None) == kvdro.KVDRO_EINVAL
    assert h.value is None


def test_host_tensors_are_refused():
    k = torch.zeros((2, 16, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        kvdro.kvdro_kv_open(None, k, k)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        kvdro.kvdro_kv_plan(None, 16, i, i, i, i[None], i, i, i, i, i, i, i)
    cache = kvdro.KvdroKv()
    cache.dtype, cache.heads, cache.head_dim, cache.handle = torch.bfloat16, 1, 64, None
    with pytest.raises(ValueError, match="CUDA"):
        kvdro.kvdro_kv_append(cache, k[0], k[0], i)
    with pytest.raises(ValueError, match="CUDA"):
        kvdro.kvdro_kv_attend(cache, k[0], i, i, i[None], k[0])


@pytest.mark.gpu
def test_refusals():
    ctx = kvdro.kvdro_create(0)

    def dev(*shape, dt=torch.bfloat16):
        return torch.zeros(shape, dtype=dt, device="cuda")

    def refused(call, *a, match="", **kw):
        with pytest.raises(kvdro.KvdroError, match=match) as e:
            call(*a, **kw)
        assert e.value.status == kvdro.KVDRO_EINVAL

    opened = kvdro.kvdro_kv_open
    for shape, match in (((2, 24, 1, 64), "page_size"), ((2, 8, 1, 64), "page_size"), ((2, 256, 1, 64), "page_size"), ((2, 16, 1, 96), "head_dim"),
                         ((2, 16, 1, 256), "head_dim"), ((1, 16, 1025, 64), "n_kv_heads")):
        refused(opened, ctx, dev(*shape), dev(*shape), match=match)
    with pytest.raises(TypeError):
        opened(ctx, dev(2, 16, 1, 64, dt=torch.float32), dev(2, 16, 1, 64, dt=torch.float32))
    with pytest.raises(ValueError):
        opened(ctx, dev(2, 16, 1, 64), dev(2, 16, 2, 64))
    with pytest.raises(ValueError):
        opened(ctx, dev(2, 16, 64, 2).transpose(2, 3), dev(2, 16, 64, 2).transpose(2, 3))
    odd = dev(2, 16, 2, 68)
    refused(opened, ctx, odd[..., :64], odd[..., :64], match="multiple of 8")
    flat = dev(2 * 16 * 64 + 1)[1:].view(2, 16, 1, 64)
    refused(opened, ctx, flat, flat, match="aligned")

    k, v = dev(4, 16, 2, 64), dev(4, 16, 2, 64)
    c = opened(ctx, k, v)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, out = dev(3, 4, 64), dev(3, 4, 64)
    args = (c, q, i(0, 3), i(3), i(0, 1)[None], out)
    att = kvdro.kvdro_kv_attend
    att(*args)
    refused(att, *args, window=5, causal=False, match="window")
    refused(att, *args, window=-1, match="window")
    refused(att, *args, scale=float("nan"), match="scale")
    refused(att, *args, softcap=-1.0, match="softcap")
    refused(att, *args, softcap=float("inf"), match="softcap")
    refused(att, *args, softcap=1001.0, match="softcap")
    refused(att, *args, softcap=1e-9, match="softcap")
    refused(att, *args, max_q=-1, match="max_q")
    lib, p = kvdro.load_library(), q.data_ptr()  # sizes that no array here has
    for T, max_pages, text in ((1 << 29, 1, "2^30"), (3, (1 << 26) + 1, "2^30"), ((1 << 30) + 1, 1, "2^30")):
        st = lib.kvdro_kv_attend(c.handle, 1, T, 4, 0, p, None, p, p, p, max_pages, 1.0, 1, 0, 0.0, p, None, None, None)
        assert st == kvdro.KVDRO_EINVAL and text in kvdro.kvdro_last_error(ctx)
    refused(att, c, dev(3, 3, 64), *args[2:5], dev(3, 3, 64), match="n_heads")
    refused(att, c, dev(3, 4, 68)[..., :64], *args[2:], match="multiple of 8")
    refused(att, *args[:5], dev(3 * 4 * 64 + 1)[1:].view(3, 4, 64), match="aligned")
    for bad in (dev(3, 4, 128), dev(2, 4, 64), dev(3, 4, 64, dt=torch.float16)):
        with pytest.raises((ValueError, TypeError)):
            att(*args[:5], bad)
    for n, bad in ((2, i(0, 1, 3)), (3, i(3, 3)), (2, i(0, 3).long())):
        with pytest.raises((ValueError, TypeError)):
            att(*args[:n], bad, *args[n + 1:])
    with pytest.raises(ValueError, match="lse"):
        att(*args, lse=dev(3, 5, dt=torch.float32))
    att(c, q[:0], i(0, 0), i(0), i(0)[None], out[:0])  # nothing to do

    app = kvdro.kvdro_kv_append
    new = dev(3, 2, 64)
    app(c, new, new, i(0, 1, -1))
    app(c, new[:0], new[:0], i())
    with pytest.raises(ValueError):
        app(c, new, new, i(0, 1))
    with pytest.raises(ValueError):
        app(c, dev(3, 3, 64), new, i(0, 1, 2))
    refused(app, c, dev(3, 2, 68)[..., :64], new, i(0, 1, 2), match="multiple of 8")

    plan = kvdro.kvdro_kv_plan
    one = lambda: i(0)  # noqa: E731
    ok = dict(cached=one(), new_len=i(1), held=one(), table=i(0)[None], ring=i(0, 1), pool=i(0, 2), held_out=one(), pool_out=i(0, 0), q_off=i(0, 0),
              kv_len=one(), slot=one())
    plan(ctx, 16, **ok)
    refused(plan, ctx, 17, **ok, match="page_size")
    refused(plan, ctx, 16, **{**ok, "held_out": ok["held"]}, match="overlaps")
    refused(plan, ctx, 16, **{**ok, "pool_out": ok["pool"]}, match="overlaps")
    for name in ("cached", "held", "pool", "q_off", "kv_len"):
        with pytest.raises(ValueError, match=name):
            plan(ctx, 16, **{**ok, name: i(0, 0, 0, 0)})
    kvdro.kvdro_sync(ctx)
    lib = kvdro.load_library()
    import numpy as np
    host = np.zeros(64, np.int32)
    assert lib.kvdro_kv_append(c.handle, 1, host.ctypes.data, None, host.ctypes.data, None, host.ctypes.data, None) == kvdro.KVDRO_EINVAL
    assert "device memory" in kvdro.kvdro_last_error(ctx)
    kvdro.kvdro_destroy(ctx)
