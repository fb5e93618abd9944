"""What bench.py does around its timed region, on the host."""

import gc

import pytest

import bench


def test_no_garbage_collection_inside_the_timed_region():
    """Objects by the hundred thousand, as an event per call leaves them, start no collection inside and may again behind it."""
    seen = []
    watch = lambda phase, info: seen.append((phase, info["generation"]))
    gc.callbacks.append(watch)
    try:
        assert gc.isenabled()
        with bench.no_collection():
            assert seen and seen[-1] == ("stop", 2)          # a full one right before
            del seen[:]
            kept = [[i] for i in range(200000)]
            assert not seen
        assert gc.isenabled()
        kept = [[i] for i in range(len(kept))]
        assert seen
    finally:
        gc.callbacks.remove(watch)


def test_collection_stays_off_where_it_was_off_and_comes_back_after_an_error():
    gc.disable()
    try:
        with bench.no_collection():
            pass
        assert not gc.isenabled()
    finally:
        gc.enable()
    with pytest.raises(ZeroDivisionError):
        with bench.no_collection():
            1 / 0
    assert gc.isenabled()
