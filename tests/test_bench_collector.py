"""What the benchmark does about Python's garbage collector before it times."""

import gc

import torch  # noqa: F401  (its objects are most of what a collection walks)

import bench


def test_a_full_collection_walks_little_after_start_up():
    try:
        bench.settle()
        assert gc.isenabled()
        assert gc.get_freeze_count() > 50 * len(gc.get_objects())
    finally:
        gc.unfreeze()
