"""Page cache calls on several streams: scratch, status and what kvdro_sync waits for."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_16892_gb300 import kvdro  # noqa: E402
from tests.kv_support import Case  # noqa: E402

A_WHILE = 500_000_000  # GPU clocks: a quarter of a second


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("lens", [[(1, 20000), (1, 300)], [(300, 4000)], [(1, 9000), (300, 3000)]], ids=["decode", "chunk", "both"])
def test_scratch_of_a_new_context_is_clear_whatever_stream_uses_it_first(lens):
    """The default stream is busy when the cache is opened, and the first call, whose rows are split over many CTAs,
    goes to a stream that is not ordered behind it."""
    case = Case(lens, "bf16", 128, 8, 2, 16, seed=1)
    first = kvdro.kvdro_create(0)  # loads the kernels
    case.check(*case.run(first))
    kvdro.kvdro_destroy(first)
    side = torch.cuda.Stream()
    for _ in range(3):
        junk = torch.full((1 << 20,), 7, dtype=torch.int32, device="cuda")  # what fresh memory may hold
        del junk
        torch.cuda.empty_cache()
        ctx = kvdro.kvdro_create(0)
        try:
            torch.cuda.synchronize()
            torch.cuda._sleep(A_WHILE)
            cache = kvdro.kvdro_kv_open(ctx, case.k, case.v)
            busy = not torch.cuda.default_stream().query()
            outs = [torch.empty_like(case.q) for _ in range(4)]
            for out in outs:
                kvdro.kvdro_kv_attend(cache, case.q, case.q_off, case.kv_len, case.table, out, stream=side)
            side.synchronize()
            assert busy, "opening a cache waited for the caller's work"
            for out in outs:
                case.check(out, None)
            kvdro.kvdro_sync(ctx)
        finally:
            kvdro.kvdro_destroy(ctx)
