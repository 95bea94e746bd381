"""The 4-bit KV cache without a GPU: the oracle's format on hand values, sizes,
and the refusals of its entry points (all before any device work; the device
pointers are never dereferenced)."""

import ctypes
from ctypes import POINTER, byref, c_int32, c_void_p

import numpy as np
import pytest

import paper_2512_04752_amd as sv
import workload as wl
from oracle import kv4 as O
from paper_2512_04752_amd import binding as B

FAKE_DEV = 0x7F0000000000
CFG = wl.TINY


def i32(*v):
    return (c_int32 * max(len(v), 1))(*v)


# ---- the oracle's format ----------------------------------------------------

def test_codes_of_hand_values():
    # 6 fixes the exponent at 0; midpoints go to the even code
    x = np.zeros(32)
    x[:12] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.26, -5.1, 0.1, -0.0]
    want = [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, -6.0, 0.0, 0.0]
    assert O.quantise(x, 32)[:12].tolist() == want


@pytest.mark.parametrize("top,e", [(0.0, -126), (6.0, 0), (6.0 + 1e-9, 1), (3.0, -1), (12.0, 1),
                                   (2.0 ** -130, -126), (2.5e38, 125), (3.3e38, 125)])
def test_exponent(top, e):
    assert O.exponent(top) == e


def test_non_finite_group_is_nan_alone():
    x = np.ones(64)
    x[40] = np.inf
    y = O.quantise(x, 32)
    assert (y[:32] == 1).all() and np.isnan(y[32:]).all()


def test_rotation_is_relative():
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(1, 1, 64)), rng.normal(size=(1, 1, 64))
    dots = [(O.rotate(q, [p + 5], 1e4) * O.rotate(k, [p], 1e4)).sum() for p in (0, 7, 30000)]
    assert np.allclose(dots, dots[0], atol=1e-9)


def test_page_decoding_by_hand():
    d = 64
    page = np.zeros(64 * (d + 2 + 2), np.uint8)
    page[64 * d:64 * d + 64 * 2] = 127                        # K scales 1
    page[64 * d + 128:].view(np.uint16)[:] = 0x4000           # V scales 2
    page[16 * d + 512 + 3 * 16 + 2] = 0x2D                    # key 35, dims 36 and 37: -3 and 1
    page[32 * d + 1 * 4 * d + (5 * 2 + 1) * 4 + 3] = 0xF1     # keys 14, 15, dim 37: 0.5 and -6
    K, V = O.decode_page(page, 1, 1, d)
    assert K[0, 0, 35, 36] == -3 and K[0, 0, 35, 37] == 1 and np.count_nonzero(K) == 2
    assert V[0, 0, 14, 37] == 1 and V[0, 0, 15, 37] == -12 and np.count_nonzero(V) == 2


# ---- sizes ------------------------------------------------------------------

def test_bytes():
    page = CFG.n_layers * CFG.n_kv_heads * 64 * (CFG.head_dim + CFG.head_dim // 32 + 2)
    assert sv.spec_kv4_page_bytes(CFG) == page
    up = lambda x: (x + 255) // 256 * 256   # noqa: E731
    assert sv.spec_kv4_bytes(CFG, 3, 5) == up(5 * page) + up(3 * 32)
    # 3.8 times the positions of the bf16 pool in the same bytes
    bf16 = sv.spec_kv_bytes(wl.LLAMA_8B, [64 * 1000])
    assert 3.7 < bf16 / sv.spec_kv4_bytes(wl.LLAMA_8B, 1, 1000) < 4
    assert sv.spec_kv4_bytes(CFG, 0, 5) == sv.spec_kv4_bytes(CFG, 3, 0) == 0
    bad = wl.ModelConfig(2, 256, 4, 2, 32, 1024, 1024)
    assert sv.spec_kv4_bytes(bad, 3, 5) == sv.spec_kv4_page_bytes(bad) == 0
    a, b = sv.spec_kv4_step_bytes(CFG, 2, 10, 4), sv.spec_kv4_step_bytes(CFG, 2, 4000, 90)
    assert 0 < a < b
    assert sv.spec_kv4_step_bytes(CFG, 3, 2, 4) == 0 == sv.spec_kv4_step_bytes(CFG, 1, 2, 0)


# ---- refusals ---------------------------------------------------------------

class Fake:
    def __init__(self, n_samples=3, n_pages=10):
        self.L = sv.lib()
        self.c = B.make_config(CFG)
        self.kv = c_void_p()
        need = sv.spec_kv4_bytes(CFG, n_samples, n_pages)
        assert self.alloc(n_samples, n_pages, FAKE_DEV, need) == 0

    def alloc(self, n, pages, dev, size, cfg=None):
        return self.L.spec_kv4_alloc(byref(cfg or self.c), n, pages, c_void_p(dev), size, byref(self.kv))

    def begin(self, ids, offsets, parents, lens, ws=FAKE_DEV, ws_bytes=1 << 30):
        self.step = c_void_p()
        (_, a), (_, b), (_, d) = (B._i32(x) for x in (ids, offsets, lens))
        p = None if parents is None else B._i32(parents)
        return self.L.spec_kv4_step_begin(self.kv, len(ids), a, b, p[1] if p else None, d, c_void_p(ws),
                                          ws_bytes, None, byref(self.step))

    def error(self):
        return self.L.spec_last_error().decode()


@pytest.fixture
def fake():
    f = Fake()
    assert f.L.spec_kv4_map(f.kv, 0, 2, i32(4, 2)) == 0
    assert f.L.spec_kv4_map(f.kv, 1, 3, i32(9, 0, 1)) == 0
    yield f
    f.L.spec_kv4_free(f.kv)


def test_alloc_refusals(fake):
    kv = fake.kv
    need = sv.spec_kv4_bytes(CFG, 3, 10)
    try:
        assert fake.alloc(3, 10, FAKE_DEV, need - 1) == -3
        assert fake.alloc(3, 10, FAKE_DEV + 128, need) == -1
        assert fake.alloc(0, 10, FAKE_DEV, need) == -1
        assert fake.alloc(3, 0, FAKE_DEV, need) == -1
        assert fake.alloc(3, 10, 0, need) == -1
        bad = B.make_config(wl.ModelConfig(2, 200, 4, 2, 64, 1024, 1024))
        assert fake.alloc(3, 10, FAKE_DEV, need, bad) == -6 and "hidden" in fake.error()
    finally:
        fake.kv = kv


@pytest.mark.parametrize("sample,pages", [(3, [0]), (-1, [0]), (0, [10]), (0, [-1]), (0, [3, 3]),
                                          (0, list(range(11)))])
def test_map_refusals(fake, sample, pages):
    assert fake.L.spec_kv4_map(fake.kv, sample, len(pages), i32(*pages)) == -1 and fake.error()
    # the tables are as they were: sample 0 holds two pages
    assert fake.begin([0], [0, 1], [-1], [127], ws_bytes=0) == -5
    assert fake.begin([0], [0, 1], [-1], [128], ws_bytes=0) == -3


TREE = [-1, 0, 0]


@pytest.mark.parametrize("case,code", [
    ("root", -2), ("after", -2), ("self", -2), ("empty", -2), ("backwards", -2), ("first", -2),
    ("big", -6), ("pages", -3), ("unmapped", -3), ("dup", -1), ("sample", -1), ("len", -1),
    ("batch", -1), ("ws", -5), ("ws_align", -1), ("ws_null", -1), ("run_pages", -3), ("run_empty", -2),
])
def test_begin_refusals(fake, case, code):
    ids, offs, par, lens, kw = [0, 1], [0, 3, 6], TREE + TREE, [10, 20], {}
    if case == "root":
        par = TREE + [0, 0, 0]
    elif case == "after":
        par = TREE + [-1, 2, 0]
    elif case == "self":
        par = TREE + [-1, 1, 0]
    elif case == "empty":
        offs, par = [0, 3, 3], TREE
    elif case == "backwards":
        offs = [0, 3, 2]
    elif case == "first":
        offs = [1, 3, 6]
    elif case == "big":
        offs, par, lens = [0, 1, 258], [-1] + [-1] + list(range(256)), [10, 0]
        fake.L.spec_kv4_map(fake.kv, 1, 5, i32(9, 0, 1, 3, 5))
    elif case == "pages":
        lens = [126, 20]
    elif case == "unmapped":
        ids = [0, 2]
    elif case == "dup":
        ids = [1, 1]
    elif case == "sample":
        ids = [0, 3]
    elif case == "len":
        lens = [10, -1]
    elif case == "batch":
        ids, offs, par, lens = [], [0], [], []
    elif case == "ws":
        kw = dict(ws_bytes=sv.spec_kv4_step_bytes(CFG, 2, 6, 2) - 1)
    elif case == "ws_align":
        kw = dict(ws=FAKE_DEV + 64)
    elif case == "ws_null":
        kw = dict(ws=0)
    elif case == "run_pages":
        par, offs, lens = None, [0, 129, 130], [0, 0]
    elif case == "run_empty":
        par, offs = None, [0, 0, 4]
    assert fake.begin(ids, offs, par, lens, **kw) == code, fake.error()
    assert fake.error() and not fake.step.value


def test_shared_pages_are_read_only(fake):
    """Pages 9 and 0 belong to samples 1 and 2: what would write there is refused."""
    L = fake.L
    assert L.spec_kv4_map(fake.kv, 2, 3, i32(9, 0, 5)) == 0
    assert fake.begin([1], [0, 1], [-1], [127], ws_bytes=0) == -1 and "page 0" in fake.error()
    assert fake.begin([1], [0, 1], [-1], [128], ws_bytes=0) == -5       # its own third page: ws is next
    dev = c_void_p(FAKE_DEV)
    assert L.spec_kv4_commit(fake.kv, 1, i32(2), i32(60), dev, dev, dev, None) == -1
    assert "page 9" in fake.error()
    assert L.spec_kv4_map(fake.kv, 2, 0, None) == 0                      # gives them back
    assert fake.begin([1], [0, 1], [-1], [127], ws_bytes=0) == -5


def test_commit_refusals(fake):
    L, dev = fake.L, c_void_p(FAKE_DEV)
    assert L.spec_kv4_commit(fake.kv, 2, i32(0, 0), i32(5, 5), dev, dev, dev, None) == -1
    assert L.spec_kv4_commit(fake.kv, 1, i32(0), i32(128), dev, dev, dev, None) == -3
    assert L.spec_kv4_commit(fake.kv, 1, i32(0), i32(-1), dev, dev, dev, None) == -3
    assert L.spec_kv4_commit(fake.kv, 1, i32(2), i32(0), dev, dev, dev, None) == -3      # no pages
    assert L.spec_kv4_commit(fake.kv, 4, i32(0, 1, 2, 3), i32(0, 0, 0, 0), dev, dev, dev, None) == -1
    assert L.spec_kv4_commit(fake.kv, 1, i32(0), i32(5), None, dev, dev, None) == -1


def test_null_handles():
    L, dev = sv.lib(), c_void_p(FAKE_DEV)
    assert L.spec_kv4_free(None) == L.spec_kv4_step_free(None) == -1
    assert L.spec_kv4_map(None, 0, 0, None) == -1
    assert L.spec_kv4_append(None, 0, dev, 128, dev, 128, 1, None) == -1
    assert L.spec_kv4_read(None, 0, dev, 128, dev, 128, None) == -1
    assert L.spec_kv4_attend(None, 0, dev, 256, dev, None) == -1
    assert ctypes.sizeof(POINTER(c_int32)) == 8


def test_largest_pool_and_run(fake):
    """Page places and row numbers are 32-bit: what would pass them is refused."""
    kv, fake.kv = fake.kv, c_void_p()
    try:
        big = B.make_config(wl.LLAMA_8B)
        page = sv.spec_kv4_page_bytes(wl.LLAMA_8B)
        most = 0xffffffff // (page // 128)
        need = sv.spec_kv4_bytes(wl.LLAMA_8B, 1, most + 1)
        assert fake.alloc(1, most + 1, FAKE_DEV, need, big) == -6 and "512 GB" in fake.error()
        # 4 query heads per KV head: rows * 16 in 32 bits
        few = B.make_config(wl.ModelConfig(1, 512, 8, 2, 64, 1024, 1024))
        assert fake.alloc(1, 1, FAKE_DEV, 1 << 30, few) == 0
        assert fake.begin([0], [0, 1 << 28], None, [0], ws_bytes=0) == -6 and "rows" in fake.error()
        assert fake.begin([0], [0, (1 << 28) - 1], None, [0], ws_bytes=0) == -3       # then its pages
    finally:
        fake.L.spec_kv4_free(fake.kv)
        fake.kv = kv


def verify(fake, ids=(0, 1), offs=(0, 3, 6), toks=(1, 2, 3, 4, 5, 6), parents=tuple(TREE + TREE), lens=(10, 20),
           ws=FAKE_DEV, ws_bytes=0, cfg=None, samp=None):
    n = CFG.n_layers
    arrays = {k: (c_void_p * n)(*[FAKE_DEV] * n) for k in B.Weights.LAYER_FIELDS}
    w = B.spec_weights(FAKE_DEV, FAKE_DEV, FAKE_DEV,
                       *[ctypes.cast(arrays[k], POINTER(c_void_p)) for k in B.Weights.LAYER_FIELDS])
    args = [B._i32(x) for x in (ids, offs, toks, parents, lens)]
    dev = c_void_p(FAKE_DEV)
    return fake.L.spec_verify_kv4(byref(cfg or fake.c), byref(w), fake.kv, len(ids), *[a[1] for a in args],
                                  c_void_p(ws), ws_bytes, None, samp, dev, dev, dev, None)


def test_verify_refusals(fake):
    assert verify(fake) == -5 and "workspace" in fake.error()             # all else is in order
    assert verify(fake, ids=(1, 1)) == -1
    assert verify(fake, ids=(0, 3)) == -1
    assert verify(fake, lens=(126, 20)) == -3                               # 128 positions, 129 needed
    assert verify(fake, lens=(-1, 20)) == -1
    assert verify(fake, parents=(-1, 0, 2, -1, 0, 0)) == -2
    assert verify(fake, parents=(0, 0, 0, -1, 0, 0)) == -2
    assert verify(fake, toks=(1, 2, CFG.vocab, 4, 5, 6)) == -2
    assert verify(fake, toks=(1, 2, -1, 4, 5, 6)) == -2
    assert verify(fake, offs=(0, 3, 3), lens=(10, 20)) == -2
    assert verify(fake, ws=FAKE_DEV + 128, ws_bytes=1 << 30) == -1
    other = B.make_config(wl.ModelConfig(CFG.n_layers, CFG.hidden, CFG.n_heads, CFG.n_kv_heads, CFG.head_dim,
                                         CFG.ffn + 128, CFG.vocab))
    assert verify(fake, cfg=other) == -1 and "config" in fake.error()
    assert fake.L.spec_kv4_map(fake.kv, 2, 1, i32(4)) == 0                  # page 4 is sample 0's too
    assert verify(fake) == -1 and "page 4" in fake.error()


def test_verify_workspace_bytes():
    one = sv.spec_workspace_bytes_kv4(CFG, 1, 8, 4)
    assert 0 < one < sv.spec_workspace_bytes_kv4(CFG, 4, 800, 40)
    assert one <= sv.spec_workspace_bytes_kv4(CFG, 1, 8, 4, sampled=True)
    assert one >= sv.spec_kv4_step_bytes(CFG, 1, 8, 4)
    for args in ((0, 8, 4), (2, 1, 4), (1, 8, 0)):
        assert sv.spec_workspace_bytes_kv4(CFG, *args) == 0
    assert sv.spec_workspace_bytes_kv4(wl.ModelConfig(2, 256, 4, 2, 32, 1024, 1024), 1, 8, 4) == 0
