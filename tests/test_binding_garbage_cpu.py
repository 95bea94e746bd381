"""The Python calls leave nothing that only a full garbage collection frees: with
torch loaded one takes some 25 ms, in which no step is enqueued."""

import gc
import weakref

import numpy as np
import pytest

import paper_2512_04752_amd as sv
import workload as wl
from paper_2512_04752_amd import binding as B


def garbage(call):
    call()
    gc.collect()
    gc.disable()
    try:
        for _ in range(50):
            call()
        return gc.collect()
    finally:
        gc.enable()


def test_arrays():
    assert garbage(lambda: B._i32([1, 2, 3])) == 0
    assert garbage(lambda: B._i32(np.arange(5, dtype=np.int32))) == 0
    assert garbage(lambda: B._i32([])) == 0


def test_calls():
    model = sv.CostModel(4.0, 1e-5, 0.01, 0.0)
    assert garbage(lambda: sv.spec_kv_bytes(wl.TINY, [64, 128])) == 0
    assert garbage(lambda: sv.spec_select_draft_count(model, [10, 20], [0, 2, 3], [-1, 0, -1],
                                                      [1.0, 0.5, 1.0], 2)) == 0
    assert garbage(lambda: B._kv4_arrays([0], [0, 2], [5], parents=[-1, 0])) == 0


@pytest.mark.parametrize("values", [[7, -3, 9], []])
def test_a_pointer_keeps_its_array(values):
    arr, p = B._i32(values)
    ref = weakref.ref(arr)
    del arr
    gc.collect()
    assert ref() is not None and p[:len(values)] == values
    del p
    assert ref() is None
