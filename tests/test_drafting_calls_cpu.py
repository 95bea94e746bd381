"""Sizes and refusals of the drafting operators, without a GPU: pointers stand in for
device memory, and every call here is refused before anything is launched."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2512_04752_amd as sv
import workload as wl
from oracle import drafting as O
from paper_2512_04752_amd import binding as B

P = 1 << 20                              # stands in for a 256-byte aligned device address
INVALID, CAPACITY, WORKSPACE, UNSUPPORTED = -1, -3, -5, -6


def test_w4_bytes():
    # row tiles of 16, column tiles of 128: 1 KB of codes each, 256 bytes of scales per four
    assert sv.spec_w4_bytes(1, 32) == 1024 + 256
    assert sv.spec_w4_bytes(17, 128) == 2 * (1024 + 256)
    assert sv.spec_w4_bytes(16, 640) == 5 * 1024 + 2 * 256
    assert sv.spec_w4_bytes(4096, 4096) == 4096 * 4096 // 2 + 4096 * 4096 // 32
    assert sv.spec_w4_bytes(1 << 24, 1 << 24) == (1 << 48) // 2 + (1 << 48) // 32
    for rows, cols in ((0, 32), (1, 0), (-1, 32), (1, -32), (1, 40), ((1 << 24) + 1, 32), (1, (1 << 24) + 32)):
        assert sv.spec_w4_bytes(rows, cols) == 0
        assert sv.spec_w4_workspace_bytes(rows, cols, 4) == 0


def test_w4_workspace_grows_with_rows():
    for rows, cols in ((16, 32), (293, 1088), (4096, 14336), (128256, 4096), (512, 1024)):
        sizes = [sv.spec_w4_workspace_bytes(rows, cols, n) for n in (1, 2, 16, 17, 64, 65, 300, 1024, 5000)]
        assert sizes == sorted(sizes) and sizes[-1] <= 256 << 20
    assert sv.spec_w4_workspace_bytes(16, 32, 0) == 0


def linear(m=(P, 48, 64), x=P, x_stride=64, n=3, out=P, out_stride=48, kind=1, ws=P, ws_bytes=1 << 30):
    m = None if m is None else ctypes.byref(B.spec_w4(*m))
    return B.lib().spec_w4_linear(m, x, x_stride, n, out, out_stride, kind, ws, ws_bytes, None)


@pytest.mark.parametrize("changed,code", [
    (dict(m=None), INVALID), (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(m=(None, 48, 64)), INVALID),
    (dict(m=(P + 128, 48, 64)), INVALID), (dict(m=(P, 0, 64)), INVALID), (dict(m=(P, 48, 40)), UNSUPPORTED),
    (dict(x=P + 8), INVALID), (dict(x_stride=63), INVALID), (dict(x_stride=68), INVALID), (dict(x_stride=56), INVALID),
    (dict(n=-1), INVALID), (dict(n=(1 << 20) + 1), UNSUPPORTED), (dict(out=P + 2), INVALID), (dict(out_stride=47), INVALID),
    (dict(x_stride=(1 << 28) + 8), UNSUPPORTED),
    (dict(m=(P, 1 << 24, 64), n=1025, out_stride=1 << 24), UNSUPPORTED), (dict(kind=0, out=P + 1), INVALID), (dict(kind=3), INVALID), (dict(kind=-1), INVALID)])
def test_linear_refusals(changed, code):
    assert linear(**changed) == code
    assert B.lib().spec_last_error()


def test_linear_of_no_rows():
    assert linear(n=0) == 0


def test_split_products_need_their_workspace():
    rows, cols, n = 1024, 8192, 128
    need = sv.spec_w4_workspace_bytes(rows, cols, n)
    call = dict(m=(P, rows, cols), x_stride=cols, n=n, out_stride=rows)
    if need:
        assert linear(**call, ws_bytes=0) == WORKSPACE
        assert linear(**call, ws=None) == WORKSPACE
        assert linear(**call, ws=P + 16) == INVALID


def test_gate_up_refusals():
    def call(gate=(P, 48, 64), up=(P, 48, 64)):
        g, u = (None if m is None else ctypes.byref(B.spec_w4(*m)) for m in (gate, up))
        return B.lib().spec_w4_gate_up(g, u, P, 64, 3, P, 48, P, 1 << 30, None)

    for bad in (dict(gate=None), dict(up=None), dict(up=(P, 32, 64)), dict(up=(P, 48, 96)), dict(up=(None, 48, 64)),
                dict(up=(P + 64, 48, 64))):
        assert call(**bad) == INVALID


def test_pack_refusals():
    def pack(w=P, stride=64, rows=48, cols=64, data=P, size=1 << 30):
        return B.lib().spec_w4_pack(w, stride, rows, cols, data, size, None)

    for bad, code in ((dict(w=None), INVALID), (dict(data=None), INVALID), (dict(data=P + 16), INVALID),
                      (dict(w=P + 4), INVALID), (dict(stride=56), INVALID), (dict(stride=65), INVALID),
                      (dict(rows=0), INVALID), (dict(cols=48), UNSUPPORTED),
                      (dict(size=sv.spec_w4_bytes(48, 64) - 1), CAPACITY)):
        assert pack(**bad) == code
    m = B.spec_w4(P, 48, 64)
    unpack = B.lib().spec_w4_unpack
    assert unpack(None, P, 64, None) == INVALID and unpack(ctypes.byref(m), P, 60, None) == INVALID
    assert unpack(ctypes.byref(m), None, 64, None) == INVALID


def test_tensors_off_the_device():
    w, data = torch.zeros(48, 64, dtype=torch.bfloat16), torch.zeros(sv.spec_w4_bytes(48, 64), dtype=torch.uint8)
    for call in (lambda: sv.spec_w4_pack(w, data), lambda: sv.spec_w4_unpack(data, w), lambda: sv.W4Matrix(w),
                 lambda: sv.spec_beam_select(torch.zeros(1, 2, 9), torch.zeros(1, 2), *[torch.zeros(1, 2).int()] * 2,
                                             torch.zeros(1, 2))):
        with pytest.raises(ValueError, match="device"):
            call()


def beam(logits=P, stride=100, bf16=0, groups=2, width=3, vocab=100, scores=P, last=None, eos=-1, k=4, parents=P,
         tokens=P, new=P, ws=P, ws_bytes=1 << 30):
    return B.lib().spec_beam_select(logits, stride, bf16, groups, width, vocab, scores, last, eos, k, parents, tokens,
                                    new, ws, ws_bytes, None)


@pytest.mark.parametrize("changed,code", [
    (dict(logits=None), INVALID), (dict(scores=None), INVALID), (dict(parents=None), INVALID), (dict(tokens=None), INVALID),
    (dict(new=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 8), INVALID), (dict(ws_bytes=64), WORKSPACE),
    (dict(stride=99), INVALID), (dict(bf16=2), INVALID), (dict(groups=0), INVALID), (dict(width=0), INVALID),
    (dict(width=65), INVALID), (dict(vocab=0), INVALID), (dict(k=0), INVALID), (dict(k=65), INVALID),
    (dict(eos=100, last=P), INVALID), (dict(eos=-2, last=P), INVALID), (dict(eos=3), INVALID), (dict(logits=P + 2), INVALID),
    (dict(bf16=1, logits=P + 1), INVALID), (dict(scores=P + 2), INVALID), (dict(groups=1 << 17, width=64), UNSUPPORTED),
    (dict(vocab=(1 << 30) + 1, stride=1 << 31), UNSUPPORTED)])
def test_beam_refusals(changed, code):
    assert beam(**changed) == code
    assert B.lib().spec_last_error()


def test_beam_workspace():
    assert sv.spec_beam_workspace_bytes(0, 1, 10, 1) == 0
    assert sv.spec_beam_workspace_bytes(1, 65, 10, 1) == 0
    for shape in ((1, 1, 1, 1), (128, 8, 128256, 8), (1, 64, 128256, 64)):
        assert 0 < sv.spec_beam_workspace_bytes(*shape) < 16 << 20
    rows = 65536 * 64                    # enough to fill the chip: one segment each, of sum, top and k candidates
    assert sv.spec_beam_workspace_bytes(65536, 64, 1000, 64) == rows * (8 + 4 + 64 * 8)


def arrays(ids, begin, end):
    out = [np.ascontiguousarray(x, dtype=np.int32) for x in (ids, begin, end)]
    return out, [x.ctypes.data for x in out]


REORDERS = [
    (dict(parents=None), INVALID), (dict(parents=P + 2), INVALID), (dict(groups=0), INVALID), (dict(width=0), INVALID),
    (dict(width=65, groups=1), INVALID), (dict(groups=3), INVALID), (dict(ids=[0, 1, 1, 3]), INVALID),
    (dict(ids=[0, 1, 2, 4]), INVALID), (dict(ids=[0, -1, 2, 3]), INVALID), (dict(begin=[-1, 0]), INVALID),
    (dict(begin=[11, 0]), INVALID), (dict(end=[10, 129]), CAPACITY)]


@pytest.mark.parametrize("changed,code", REORDERS)
def test_reorder_refusals(changed, code):
    cfg = wl.TINY
    a = dict(groups=2, width=2, ids=[0, 1, 2, 3], begin=[0, 5], end=[10, 10], parents=P)
    a.update(changed)
    kept, (ids, begin, end) = arrays(a["ids"], a["begin"], a["end"])
    L = B.lib()
    caps = (ctypes.c_int32 * 4)(128, 128, 128, 128)
    h = ctypes.c_void_p()
    c = B.make_config(cfg)
    assert L.spec_kv_alloc(ctypes.byref(c), 4, caps, P, 1 << 40, ctypes.byref(h)) == 0
    assert L.spec_kv_reorder(h, a["groups"], a["width"], ids, begin, end, a["parents"], None) == code
    assert L.spec_kv_reorder(None, 2, 2, ids, begin, end, P, None) == INVALID
    L.spec_kv_free(h)
    assert L.spec_kv4_alloc(ctypes.byref(c), 4, 8, P, 1 << 40, ctypes.byref(h)) == 0
    for s in range(4):
        assert L.spec_kv4_map(h, s, 2, (ctypes.c_int32 * 2)(2 * s, 2 * s + 1)) == 0
    call = (a["groups"], a["width"], ids, begin, end, a["parents"])
    assert L.spec_kv4_reorder(h, *call, P, 1 << 20, None) == code
    if code == CAPACITY:                 # another sample's page too; the right workspace only
        kept, (ids, begin, end) = arrays([0, 1, 2, 3], [0, 64], [64, 65])
        assert L.spec_kv4_reorder(h, 2, 2, ids, begin, end, P, P + 16, 1 << 20, None) == INVALID
        assert L.spec_kv4_map(h, 3, 2, (ctypes.c_int32 * 2)(6, 5)) == 0      # page 5: position 64 .. of sample 2
        assert L.spec_kv4_reorder(h, 2, 2, ids, begin, end, P, P, 1 << 20, None) == INVALID
        assert b"mapped to 2" in L.spec_last_error()
    L.spec_kv4_free(h)


def test_kv4_reorder_workspace():
    """Small calls' descriptors go along as kernel arguments; others need room for theirs."""
    L, h, c = B.lib(), ctypes.c_void_p(), B.make_config(wl.TINY)
    n = 140
    assert L.spec_kv4_alloc(ctypes.byref(c), n, 10 * n, P, 1 << 40, ctypes.byref(h)) == 0
    size = L.spec_kv4_reorder_bytes
    assert size(h, 2, 2, 10) == size(h, 64, 1, 19) == 0
    assert size(h, 65, 1, 1) == 1280 + 512
    assert size(h, 100, 8, 100) == 1792 + 100 * 8 * 100 * 4
    for bad in ((None, 1, 1, 1), (h, 0, 1, 1), (h, 1, 0, 1), (h, 1, 65, 1), (h, 1, 1, 0)):
        assert size(*bad) == 0
    for s in range(n):
        assert L.spec_kv4_map(h, s, 10, (ctypes.c_int32 * 10)(*range(10 * s, 10 * s + 10))) == 0
    kept, (ids, begin, end) = arrays(range(n), [0] * 7, [640] * 7)
    need = size(h, 7, 20, 10)
    assert need >= 256 + 7 * 20 * 10 * 4
    for ws, nbytes in ((None, 1 << 20), (P, 256)):
        assert L.spec_kv4_reorder(h, 7, 20, ids, begin, end, P, ws, nbytes, None) == WORKSPACE
    L.spec_kv4_free(h)


# ---- the oracle itself -------------------------------------------------------

def test_oracle_quantise_by_hand():
    w = np.zeros((1, 32))
    w[0, :6] = [6.0, -1.25, 0.25, 5.0, 0.75, 1.75]     # e = 0: ties go to 1, 0, 4, 1, 2
    assert O.quantise(w)[0, :6].tolist() == [6.0, -1.0, 0.0, 4.0, 1.0, 2.0]
    w[0, 0] = 6.01                                      # e = 1
    assert O.quantise(w)[0, :6].tolist() == [6.0, -1.0, 0.0, 4.0, 1.0, 2.0]
    w[0, 0] = 13.0                                      # e = 2
    assert O.quantise(w)[0, :4].tolist() == [12.0, -2.0, 0.0, 4.0]


def test_oracle_select_by_hand():
    z = np.log(np.array([[[0.5, 0.3, 0.2], [0.1, 0.1, 0.8]]]))
    p, t, s = O.select(z, np.log([[0.5, 0.5]]), 4)
    assert p.tolist() == [[1, 0, 0, 0]] and t.tolist() == [[2, 0, 1, 2]]
    assert np.allclose(np.exp(s), [[0.4, 0.25, 0.15, 0.1]])
    p, t, s = O.select(z, [[0.0, -5.0]], 4, [[0, 1]], 1)
    assert p.tolist() == [[0, 0, 0, 1]] and t.tolist() == [[0, 1, 2, 1]] and s[0, 3] == -5.0
    p, t, s = O.select(z, [[-np.inf, np.nan]], 2)
    assert p.tolist() == [[-1, -1]] and np.isneginf(s).all()


# ---- the verify step with weights in 4 bits ------------------------------------

class FakeStep:
    """spec_verify_w4 with pointers that stand in for device memory."""

    def __init__(self, cfg=wl.TINY, n=3):
        self.cfg, self.c, self.L = cfg, B.make_config(cfg), B.lib()
        self.kv, self.kv4 = ctypes.c_void_p(), ctypes.c_void_p()
        assert self.L.spec_kv_alloc(ctypes.byref(self.c), n, (ctypes.c_int32 * n)(*[100] * n), P, 1 << 40,
                                    ctypes.byref(self.kv)) == 0
        assert self.L.spec_kv4_alloc(ctypes.byref(self.c), n, 2 * n, P, 1 << 40, ctypes.byref(self.kv4)) == 0
        for s in range(n):
            assert self.L.spec_kv4_map(self.kv4, s, 2, (ctypes.c_int32 * 2)(2 * s, 2 * s + 1)) == 0
        q, kv, layers = cfg.n_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim, cfg.n_layers
        shapes = dict(wqkv=(q + 2 * kv, cfg.hidden), wo=(cfg.hidden, q), w_gate=(cfg.ffn, cfg.hidden),
                      w_up=(cfg.ffn, cfg.hidden), w_down=(cfg.hidden, cfg.ffn))
        self.m = {k: (B.spec_w4 * layers)(*[B.spec_w4(P, *shape)] * layers) for k, shape in shapes.items()}
        self.norms = (ctypes.c_void_p * layers)(*[P] * layers)
        self.w = B.spec_weights_w4(P, P, B.spec_w4(P, cfg.vocab, cfg.hidden), self.norms, self.m["wqkv"],
                                   self.m["wo"], self.norms, self.m["w_gate"], self.m["w_up"], self.m["w_down"])

    def call(self, kv=True, kv4=False, w=True, tokens=(5, 6, 7), parents=(-1, 0, 0), length=10, ws=P, ws_bytes=None,
             outs=P, sample=1):
        if ws_bytes is None:
            ws_bytes = sv.spec_workspace_bytes_w4(self.cfg, 1, len(tokens), 2 if kv4 else 0)
        kept, (ids, offs, toks, pars, lens) = zip(*map(B._i32, ([sample], [0, len(tokens)], tokens, parents, [length])))
        return self.L.spec_verify_w4(ctypes.byref(self.c), ctypes.byref(self.w) if w else None,
                                     self.kv if kv else None, self.kv4 if kv4 else None, 1, ids, offs, toks, pars,
                                     lens, ws, ws_bytes, None, None, outs, P, P, None)

    def close(self):
        self.L.spec_kv_free(self.kv)
        self.L.spec_kv4_free(self.kv4)


@pytest.fixture
def step():
    f = FakeStep()
    yield f
    f.close()


@pytest.mark.parametrize("changed,code", [
    (dict(w=False), INVALID), (dict(kv=False), INVALID), (dict(kv4=True), INVALID), (dict(outs=None), INVALID),
    (dict(ws=None), INVALID), (dict(ws=P + 16), INVALID), (dict(ws_bytes=1 << 20), WORKSPACE),
    (dict(sample=3), INVALID), (dict(length=98), CAPACITY), (dict(length=-1), INVALID),
    (dict(tokens=(5, 6, wl.TINY.vocab)), -2), (dict(parents=(-1, 1, 0)), -2), (dict(parents=(0, 0, 0)), -2),
    (dict(kv=False, kv4=True, length=126), CAPACITY), (dict(kv=False, kv4=True, ws=P + 16), INVALID),
    (dict(kv=False, kv4=True, tokens=(-1, 6, 7)), -2)])
def test_w4_step_refusals(step, changed, code):
    assert step.call(**changed) == code
    assert B.lib().spec_last_error()


@pytest.mark.parametrize("name", ["lm_head", "wqkv", "wo", "w_gate", "w_up", "w_down"])
@pytest.mark.parametrize("field,value", [("data", None), ("data", P + 16), ("rows", 16), ("cols", 32)])
def test_w4_step_refuses_matrices(step, name, field, value):
    setattr(step.w.lm_head if name == "lm_head" else step.m[name][step.cfg.n_layers - 1], field, value)
    assert step.call() == INVALID
    assert name.encode() in B.lib().spec_last_error()


def test_w4_step_refuses_missing_arrays(step):
    for name in ("tok_embed", "final_norm", "attn_norm", "wqkv", "wo", "ffn_norm", "w_gate", "w_up", "w_down"):
        kept = bytes(step.w)
        setattr(step.w, name, None)
        assert step.call() == INVALID and b"null" in B.lib().spec_last_error()
        ctypes.memmove(ctypes.byref(step.w), kept, len(kept))
    step.norms[1] = None
    assert step.call() == INVALID and b"layer 1" in B.lib().spec_last_error()


def test_w4_step_workspace():
    size = sv.spec_workspace_bytes_w4
    for pages in (0, 40):
        got = [size(wl.TINY, b, n, pages) for b, n in ((1, 1), (1, 2), (4, 16), (4, 300), (64, 5000))]
        assert got == sorted(got) and got[0] > 0
        assert size(wl.TINY, 4, 16, pages, True) > size(wl.TINY, 4, 16, pages)
    for bad in ((0, 1, 0), (2, 1, 0), (1, 1, -1)):
        assert size(wl.TINY, *bad) == 0
    # what a step sets aside for partial sums is enough for any product
    for rows, cols in ((16, 32), (6144, 4096), (4096, 14336), (14336, 4096), (128256, 4096), (1 << 20, 1 << 16)):
        assert sv.spec_w4_workspace_bytes(rows, cols, 5000) <= 64 << 20
