"""The scratch that a cache's attend calls share, with CPU tensors in the place of the GPU's."""
import gc
import weakref

import pytest
import torch

from tests.test_cache_host import cache_of, ctx, half  # noqa: F401


@pytest.fixture
def counted(ctx):  # noqa: F811
    """(context, living scratch, calls): scratch grows with the rows, as a call's does."""
    living, calls, empty = weakref.WeakSet(), [], ctx.empty

    def tracked(shape, dtype):
        t = empty(shape, dtype)
        if dtype == torch.uint8:
            living.add(t)
        return t
    ctx.empty = tracked

    class Lib:
        def dcnn_cache_scratch_bytes(self, dtype, rows, *sizes):
            return 4096 + 1000 * rows

        def dcnn_cache_attend(self, handle, a):
            calls.append((a.rows, a.scratch, a.scratch_bytes))
            gc.collect()
            assert any(t.data_ptr() == a.scratch and t.numel() >= a.scratch_bytes >= 4096 + 1000 * a.rows for t in living), "scratch that nobody holds"
            return 0
    ctx.lib = Lib()
    return ctx, living, calls


def test_eager_calls_of_rising_sizes_hold_one_scratch(counted):
    own, living, calls = counted
    cache = cache_of(own)
    for rows in range(1, 400):
        cache.attend(half(rows, 256))
    gc.collect()
    assert len(living) == 1 and cache._scratch_at[1] <= 2 * (4096 + 399000)
    assert len({at for _, at, _ in calls}) < 20                    # (made anew now and then only)
    before = len(calls)
    cache.attend(half(1, 256))
    assert calls[before][1:] == cache._scratch_at


def test_scratch_of_captured_calls(counted):
    """What a graph holds the address of is kept; what a capture makes is the graph's."""
    own, living, calls = counted
    cache = cache_of(own)
    cache.attend(half(10, 256))
    first = cache._scratch_at
    own.capturing = lambda: True
    cache.attend(half(5, 256))
    cache.attend(half(7, 256))
    cache.attend(half(300, 256))
    assert [at for _, at, _ in calls[1:3]] == [first[0]] * 2 and calls[3][2] >= 4096 + 300000 and cache._scratch_at == first
    gc.collect()
    assert len(living) == 1                                        # (the capture's own is out of the graph's memory, which the graph holds)
    own.capturing = lambda: False
    for rows in (50, 200, 390):
        cache.attend(half(rows, 256))
    gc.collect()
    assert sorted(t.numel() for t in living)[0] == first[1] and len(living) == 2 and any(t.data_ptr() == first[0] for t in living)
    own.capturing = lambda: True
    cache.attend(half(390, 256))
    own.capturing = lambda: False
    cache.attend(half(2000, 256))
    gc.collect()
    assert len(living) == 3


def test_a_cache_that_only_graphs_use_holds_nothing(counted):
    own, living, calls = counted
    cache = cache_of(own)
    own.capturing = lambda: True
    for rows in (1, 30, 20):
        cache.attend(half(rows, 256))
    gc.collect()
    assert len(living) == 0 and cache._scratch is None and len(calls) == 3
