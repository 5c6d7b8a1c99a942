"""Waits that run out in the kernel that reads prefixes in front of the requests' own tokens."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv8_support import Shared  # noqa: E402

B, PREFIX, PAGE, HKV, D = 40, 1600, 16, 2, 128


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = kvdro.kvdro_create(0)
    yield c
    kvdro.kvdro_destroy(c)


@pytest.mark.parametrize("skip", [0, 1, 2])
@pytest.mark.parametrize("bits,Hq", [(16, 8), (16, 24), (8, 8), (8, 24), (8, 48)])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(monkeypatch, ctx, bits, Hq, skip):
    """Every CTA leaves one copy out, so nothing completes its barrier, and the bounded wait for it (1 ms under the hook) gives up.  Each request
    reads its prefix where the tables' key elements, times the groups of eight rows, are 48 M at most: the prefix's table has no wider rows
    than it needs."""
    s = Shared([(1, 300)] * B, [0, B], [PREFIX], bits=bits, dtype="bf16", D=D, Hq=Hq, Hkv=HKV, page=PAGE, seed=1)
    s.prefix_table = s.prefix_table[:, :PREFIX // PAGE].contiguous()
    assert B * PREFIX * HKV * D * -(-Hq // HKV // 8) <= 48 << 20 and Hq // HKV <= 32
    monkeypatch.setenv("KVDRO_TEST_SKIP_CHUNK", str(skip))
    broken = kvdro.kvdro_create(0)
    monkeypatch.delenv("KVDRO_TEST_SKIP_CHUNK")
    try:
        for _ in range(2):
            s.run(broken)
            with pytest.raises(kvdro.KvdroError) as e:
                kvdro.kvdro_sync(broken)
            assert e.value.status == kvdro.KVDRO_ETIMEOUT
        kvdro.kvdro_sync(broken)
    finally:
        kvdro.kvdro_destroy(broken)
    s.check(*s.run(ctx))
    kvdro.kvdro_sync(ctx)
