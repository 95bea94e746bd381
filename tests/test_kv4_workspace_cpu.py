"""Workspace of a step over the 4-bit cache: what the step needs, not what the
largest one would."""

import numpy as np

import paper_2512_04752_amd as sv
import workload as wl


def test_small_steps_take_little():
    """One row behind 580 keys (10 pages, 2 key ranges at most): 8 KV heads x 2 x 16 rows of fp32 partial
    results, 131 KB, and descriptors."""
    assert sv.spec_kv4_step_bytes(wl.LLAMA_8B, 1, 1, 10) < 1 << 19
    assert sv.spec_kv4_step_bytes(wl.LLAMA_1B, 1, 1, 10) < 1 << 19
    # 4 trees of 64 nodes at 25K keys fill the table of partial tiles
    assert sv.spec_kv4_step_bytes(wl.LLAMA_8B, 4, 256, 1600) > 8192 * 16 * 128 * 4


def test_bytes_grow_with_every_argument():
    """A workspace of the largest step serves the smaller ones."""
    rng = np.random.default_rng(0)
    for _ in range(300):
        batch = int(rng.integers(1, 200))
        rows, pages = batch + int(rng.integers(0, 2000)), int(rng.integers(1, 4000))
        for cfg in (wl.TINY, wl.LLAMA_1B, wl.LLAMA_8B):
            need = sv.spec_kv4_step_bytes(cfg, batch, rows, pages)
            for a in ((batch, rows + 1, pages), (batch, rows, pages + 1), (batch + 1, rows + 1, pages),
                      (2 * batch, 2 * rows, 2 * pages)):
                assert sv.spec_kv4_step_bytes(cfg, *a) >= need
