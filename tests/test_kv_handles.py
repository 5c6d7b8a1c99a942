"""Page cache handles are closed once, never after their context and never two at a time, whoever drops them: against a fake of
the library, without a GPU."""

import gc
import threading
import time

import pytest

torch = pytest.importorskip("torch")

from paper_2607_16892_gb300 import kvdro  # noqa: E402


class Library:
    """Counts handles, and calls that run at the same time."""

    def __init__(self):
        self.open, self.next, self.inside, self.most, self.wrong, self.destroyed = set(), 1000, 0, 0, [], 0

    def _run(self, what, seconds=0.0005):
        self.inside += 1
        self.most = max(self.most, self.inside)
        time.sleep(seconds)  # another thread's turn
        what()
        self.inside -= 1
        return 0

    def kvdro_kv_open(self, ctx, out, *rest):
        def go():
            self.next += 1
            self.open.add(self.next)
            out._obj.value = self.next
        return self._run(go)

    def kvdro_kv_close(self, h):
        def go():
            if h.value in self.open:
                self.open.remove(h.value)
            else:
                self.wrong.append(h.value)
        return self._run(go)

    def kvdro_destroy(self, ctx):
        def go():
            self.destroyed += 1
            self.open.clear()
        return self._run(go, 0.02)


class Pages:
    """As much of a CUDA tensor as opening a cache looks at."""

    is_cuda, dtype, shape = True, torch.bfloat16, (2, 16, 1, 64)

    def dim(self):
        return 4

    def stride(self, i):
        return (1024, 64, 64, 1)[i]

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def lib(monkeypatch):
    fake = Library()
    monkeypatch.setattr(kvdro, "load_library", lambda *a: fake)
    monkeypatch.setattr(kvdro, "_lib_kv", None)
    yield fake
    gc.collect()


def open_cache(ctx=5):
    return kvdro.kvdro_kv_open(ctx, Pages(), Pages())


def test_a_handle_is_closed_once(lib):
    a, b = open_cache(), open_cache()
    kvdro.kvdro_kv_close(a)
    kvdro.kvdro_kv_close(a)
    del a
    assert len(lib.open) == 1
    kvdro.kvdro_destroy(5)
    assert b.handle is None and b.k is None and not lib.open
    del b
    assert lib.destroyed == 1 and not lib.wrong


def test_caches_dropped_by_several_threads_are_closed_one_at_a_time(lib):
    caches = [[open_cache() for _ in range(20)] for _ in range(4)]
    threads = [threading.Thread(target=c.clear) for c in caches]
    for t in threads:
        t.start()
    more = [open_cache() for _ in range(10)]
    for t in threads:
        t.join()
    assert lib.most == 1 and len(lib.open) == len(more) and not lib.wrong
    kvdro.kvdro_destroy(5)


def test_a_cache_dropped_while_its_context_goes(lib):
    for _ in range(5):
        caches = [open_cache() for _ in range(6)]
        t = threading.Thread(target=caches.clear)
        t.start()
        kvdro.kvdro_destroy(5)
        t.join()
        assert lib.most == 1 and not lib.wrong and not lib.open


def test_a_cycle_whose_other_part_destroys_the_context(lib):
    """The collector clears weak references before it runs finalizers, in an order of its own."""
    class Server:
        def __del__(self):
            kvdro.kvdro_destroy(5)
    gc.collect()
    gc.disable()
    try:
        s = Server()
        s.cache = [open_cache(), s]
        del s
    finally:
        gc.enable()
    gc.collect()
    assert lib.destroyed == 1 and not lib.wrong


def test_a_stale_cache_does_not_close_another_contexts_handle(lib):
    """Addresses come again: a context and a handle of the same numbers as the ones that were freed."""
    gc.disable()
    try:
        old = open_cache()
        old.owner.caches.discard(old)  # as a collector leaves it
        kvdro.kvdro_destroy(5)
        lib.next = 1000
        new = open_cache()
        assert new.handle.value == old.handle.value
        del old
        assert lib.open == {new.handle.value}
    finally:
        gc.enable()
    kvdro.kvdro_destroy(5)
