"""What the calls on caches of 8 bits, reads and shared prefixes refuse without a GPU, and the plain quantiser that the GPU tests use."""

import ctypes

import pytest

from paper_2607_16892_gb300 import kvdro

torch = pytest.importorskip("torch")

from tests.kv8_support import F64, nearest_code, quantise, two  # noqa: E402


def test_null_handles_are_refused():
    lib, h = kvdro.load_library(), ctypes.c_void_p(5)
    assert lib.kvdro_kv_open8(None, ctypes.byref(h), 0, 1, 16, 1, 64, *[None] * 6) == kvdro.KVDRO_EINVAL and h.value is None
    assert lib.kvdro_kv_read(None, 1, 1, None, None, None, 1, *[None] * 5) == kvdro.KVDRO_EINVAL
    assert lib.kvdro_kv_attend_shared(None, 1, 1, 1, 1, *[None] * 5, 1, 1, *[None] * 3, 1, 1.0, 1, 0.0, *[None] * 4, 0, None) == kvdro.KVDRO_EINVAL
    assert lib.kvdro_kv_shared_bytes(1, 8, 128, None) == kvdro.KVDRO_EINVAL
    n = ctypes.c_size_t()
    assert lib.kvdro_kv_shared_bytes(7, 8, 64, ctypes.byref(n)) == kvdro.KVDRO_OK and n.value == 7 * 8 * 66 * 4


def test_host_tensors_are_refused():
    codes, e = torch.zeros((2, 16, 1, 64), dtype=torch.float8_e4m3fn), torch.zeros((2, 1, 16), dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        kvdro.kvdro_kv_open8(None, codes, codes, e, e, torch.bfloat16)
    i, rows = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    cache = kvdro.KvdroKv()
    cache.dtype, cache.heads, cache.head_dim, cache.handle = torch.bfloat16, 1, 64, None
    with pytest.raises(ValueError, match="CUDA"):
        kvdro.kvdro_kv_read(cache, i, i, i[None], rows, rows)
    with pytest.raises(ValueError, match="CUDA"):
        kvdro.kvdro_kv_attend_shared(cache, rows, i, i, i[None], i, i, i[None], rows)


def test_the_plain_quantiser_rounds_to_the_nearest_code():
    """Against every code: the nearest, and of two as near the even one."""
    every = torch.arange(0x7f, dtype=torch.uint8).view(torch.float8_e4m3fn).to(F64)
    y = torch.cat([every, (every[1:] + every[:-1]) / 2, torch.linspace(0, 448, 4001, dtype=F64)])
    far = (y[:, None] - every).abs()
    best = far.amin(1, keepdim=True)
    ties = far == best
    even = torch.arange(0x7f) % 2 == 0
    pick = torch.where(ties.sum(1) > 1, (ties & even).to(torch.int32).argmax(1), ties.to(torch.int32).argmax(1))
    assert torch.equal(nearest_code(y), every[pick]) and torch.equal(nearest_code(-y), -every[pick])


def test_the_plain_quantiser_takes_the_least_scale():
    for top, e in ((448.0, 0), (450.0, 1), (0.0, -126), (3.0e38, 120), (224.0, -1), (226.0, 0), (2.0 ** -133, -126)):
        x = torch.zeros((1, 64), dtype=torch.bfloat16)
        x[0, 5] = top
        c, got = quantise(x)
        assert int(got) == e and float(c.abs().max()) <= 448
    h = torch.full((1, 64), 65504.0, dtype=torch.float16)
    c, e = quantise(h)
    assert float((c * two(e)[..., None])[0, 0]) == 61440.0
