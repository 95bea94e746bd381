"""ctypes binding of libspecverify.so: the C entry points under the same
names, marshalling torch tensors, numpy arrays and Python lists into
pointers.  Every step of the verify computation runs in the library's HIP
kernels; PyTorch only provides device memory and the stream.
"""

from __future__ import annotations

import contextlib
import ctypes
import functools
import os
from ctypes import POINTER, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import numpy as np
import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspecverify.so")

SPEC_MAX_TREE = 256
SPEC_ANC_WORDS = SPEC_MAX_TREE // 64   # 64-bit words of one node's ancestor set
STATUS = {0: "SPEC_OK", -1: "SPEC_ERR_INVALID", -2: "SPEC_ERR_TREE", -3: "SPEC_ERR_CAPACITY",
          -5: "SPEC_ERR_WORKSPACE", -6: "SPEC_ERR_UNSUPPORTED", -7: "SPEC_ERR_HIP"}
KERNEL_CLASS = {"gemm_qkv": 0, "attention": 1, "gemm_o": 2, "gemm_gate_up": 3, "gemm_down": 4,
                "lm_head": 5, "commit": 6, "accept": 8}   # the kernel classes of one verify step
TRANSFER_CLASS = 7                                    # spec_kv_pack / spec_kv_unpack
KV4_APPEND_CLASS = 9                                  # spec_kv4_append
OPERATOR_CLASS = {"transfer": TRANSFER_CLASS, "kv4_append": KV4_APPEND_CLASS, "w4": 10, "beam": 11, "reorder": 12}

# Every symbol the public header declares.
EXPORTS = ("spec_kv_bytes", "spec_kv_alloc", "spec_kv_free", "spec_kv_sample_layout",
           "spec_workspace_bytes", "spec_verify", "spec_kv_commit", "spec_last_error",
           "spec_profile_begin", "spec_profile_end", "spec_kv_transfer_bytes", "spec_kv_pack",
           "spec_kv_unpack", "spec_cost_model_create", "spec_cost_model_free", "spec_cost_predict",
           "spec_cost_model_stats", "spec_select_draft_count", "spec_workspace_bytes_sampled",
           "spec_verify_sampled", "spec_verify_noalloc", "spec_gemm_plan", "spec_kv4_page_bytes",
           "spec_kv4_bytes", "spec_kv4_alloc", "spec_kv4_free", "spec_kv4_map",
           "spec_kv4_step_bytes", "spec_kv4_step_begin", "spec_kv4_step_free", "spec_kv4_append",
           "spec_kv4_read", "spec_kv4_attend", "spec_kv4_commit",
           "spec_workspace_bytes_kv4", "spec_verify_kv4", "spec_workspace_bytes_w4",
           "spec_verify_w4", "spec_w4_bytes", "spec_w4_pack", "spec_w4_unpack",
           "spec_w4_workspace_bytes", "spec_w4_product_bytes", "spec_w4_linear", "spec_w4_gate_up",
           "spec_beam_workspace_bytes", "spec_beam_select", "spec_kv_reorder",
           "spec_kv4_reorder_bytes", "spec_kv4_reorder")
SPEC_KV4_PAGE = 64                # positions per page of the 4-bit pool
SPEC_NOALLOC_SCRATCH_BYTES = 320 << 20
SPEC_MAX_BEAMS = 64               # beams of a group, and continuations of a choice
SPEC_W4_BF16, SPEC_W4_F32, SPEC_W4_ADD = 0, 1, 2      # outputs of spec_w4_linear


class SpecError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class spec_model_config(ctypes.Structure):
    _fields_ = [("n_layers", c_int32), ("hidden", c_int32), ("n_heads", c_int32),
                ("n_kv_heads", c_int32), ("head_dim", c_int32), ("ffn", c_int32),
                ("vocab", c_int32), ("rope_theta", c_float), ("rms_eps", c_float)]


class spec_weights(ctypes.Structure):
    _fields_ = [("tok_embed", c_void_p), ("final_norm", c_void_p), ("lm_head", c_void_p),
                ("attn_norm", POINTER(c_void_p)), ("wq", POINTER(c_void_p)),
                ("wk", POINTER(c_void_p)), ("wv", POINTER(c_void_p)), ("wo", POINTER(c_void_p)),
                ("ffn_norm", POINTER(c_void_p)), ("w_gate", POINTER(c_void_p)),
                ("w_up", POINTER(c_void_p)), ("w_down", POINTER(c_void_p))]


class spec_cost_coeffs(ctypes.Structure):
    _fields_ = [("c0", ctypes.c_double), ("c_seq", ctypes.c_double), ("c_draft", ctypes.c_double),
                ("c_tree", ctypes.c_double), ("bucket_ratio", ctypes.c_double)]


class spec_sampling(ctypes.Structure):
    _fields_ = [("temperature", c_float), ("eos_token", c_int32), ("draft_probs", c_void_p),
                ("uniforms", c_void_p)]


class spec_w4(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("rows", c_int32), ("cols", c_int32)]


class spec_weights_w4(ctypes.Structure):
    _fields_ = [("tok_embed", c_void_p), ("final_norm", c_void_p), ("lm_head", spec_w4),
                ("attn_norm", POINTER(c_void_p)), ("wqkv", POINTER(spec_w4)), ("wo", POINTER(spec_w4)),
                ("ffn_norm", POINTER(c_void_p)), ("w_gate", POINTER(spec_w4)), ("w_up", POINTER(spec_w4)),
                ("w_down", POINTER(spec_w4))]


class spec_debug(ctypes.Structure):
    _fields_ = [("logits", c_void_p), ("argmax", c_void_p), ("depth", c_void_p),
                ("pos", c_void_p), ("anc", c_void_p)]


_lib = None


def lib():
    """Load the library; fails loudly when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing; build it with "
                           "`python -m paper_2512_04752_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    i32p = POINTER(c_int32)
    L.spec_kv_bytes.argtypes = [POINTER(spec_model_config), c_int32, i32p]
    L.spec_kv_bytes.restype = c_size_t
    L.spec_kv_alloc.argtypes = [POINTER(spec_model_config), c_int32, i32p, c_void_p, c_size_t,
                                POINTER(c_void_p)]
    L.spec_kv_free.argtypes = [c_void_p]
    L.spec_kv_sample_layout.argtypes = [c_void_p, c_int32, POINTER(c_int64), i32p]
    L.spec_workspace_bytes.argtypes = [POINTER(spec_model_config), c_int32, c_int32]
    L.spec_workspace_bytes.restype = c_size_t
    L.spec_verify.argtypes = [POINTER(spec_model_config), POINTER(spec_weights), c_void_p,
                              c_int32, i32p, i32p, i32p, i32p, i32p, c_void_p, c_size_t,
                              c_void_p, c_void_p, c_void_p, c_void_p, POINTER(spec_debug)]
    L.spec_kv_commit.argtypes = [c_void_p, c_int32, i32p, i32p, c_void_p, c_void_p, c_void_p,
                                 c_void_p]
    L.spec_workspace_bytes_sampled.argtypes = [POINTER(spec_model_config), c_int32, c_int32]
    L.spec_workspace_bytes_sampled.restype = c_size_t
    L.spec_verify_sampled.argtypes = [POINTER(spec_model_config), POINTER(spec_weights), c_void_p,
                                      c_int32, i32p, i32p, i32p, i32p, i32p, c_void_p, c_size_t,
                                      c_void_p, POINTER(spec_sampling), c_void_p, c_void_p,
                                      c_void_p, POINTER(spec_debug)]
    L.spec_verify_noalloc.argtypes = [POINTER(spec_model_config), POINTER(spec_weights),
                                      c_void_p, c_int32, i32p, i32p, i32p, i32p, i32p, c_void_p,
                                      c_void_p, c_void_p, c_void_p, POINTER(spec_debug)]
    L.spec_kv_transfer_bytes.argtypes = [c_void_p, c_int32, i32p, i32p]
    L.spec_kv_transfer_bytes.restype = c_size_t
    L.spec_kv_pack.argtypes = [c_void_p, c_int32, i32p, i32p, i32p, c_void_p, c_size_t, c_void_p]
    L.spec_kv_unpack.argtypes = [c_void_p, c_int32, i32p, i32p, i32p, c_void_p, c_size_t, c_void_p]
    L.spec_cost_model_create.argtypes = [POINTER(spec_cost_coeffs), POINTER(c_void_p)]
    L.spec_cost_model_free.argtypes = [c_void_p]
    L.spec_cost_predict.argtypes = [c_void_p, c_int64, c_int64, c_int64]
    L.spec_cost_predict.restype = ctypes.c_double
    L.spec_cost_model_stats.argtypes = [c_void_p, POINTER(c_int64), POINTER(c_int64)]
    L.spec_select_draft_count.argtypes = [c_void_p, c_int32, i32p, i32p, i32p,
                                          POINTER(c_float), c_int32, c_int32, i32p, i32p,
                                          POINTER(ctypes.c_double)]
    L.spec_last_error.restype = ctypes.c_char_p
    L.spec_profile_begin.argtypes = [c_int32, c_int32]
    L.spec_profile_end.argtypes = [POINTER(c_float), i32p]
    L.spec_gemm_plan.argtypes = [POINTER(spec_model_config), c_int32, c_int32, i32p, i32p, i32p]
    L.spec_kv4_page_bytes.argtypes = [POINTER(spec_model_config)]
    L.spec_kv4_page_bytes.restype = c_size_t
    L.spec_kv4_bytes.argtypes = [POINTER(spec_model_config), c_int32, c_int32]
    L.spec_kv4_bytes.restype = c_size_t
    L.spec_kv4_alloc.argtypes = [POINTER(spec_model_config), c_int32, c_int32, c_void_p, c_size_t,
                                 POINTER(c_void_p)]
    L.spec_kv4_free.argtypes = [c_void_p]
    L.spec_kv4_map.argtypes = [c_void_p, c_int32, c_int32, i32p]
    L.spec_kv4_step_bytes.argtypes = [POINTER(spec_model_config), c_int32, c_int32, c_int32]
    L.spec_kv4_step_bytes.restype = c_size_t
    L.spec_kv4_step_begin.argtypes = [c_void_p, c_int32, i32p, i32p, i32p, i32p, c_void_p, c_size_t,
                                      c_void_p, POINTER(c_void_p)]
    L.spec_kv4_step_free.argtypes = [c_void_p]
    L.spec_kv4_append.argtypes = [c_void_p, c_int32, c_void_p, c_int64, c_void_p, c_int64, c_int32,
                                  c_void_p]
    L.spec_kv4_read.argtypes = [c_void_p, c_int32, c_void_p, c_int64, c_void_p, c_int64, c_void_p]
    L.spec_kv4_attend.argtypes = [c_void_p, c_int32, c_void_p, c_int64, c_void_p, c_void_p]
    L.spec_kv4_commit.argtypes = [c_void_p, c_int32, i32p, i32p, c_void_p, c_void_p, c_void_p,
                                  c_void_p]
    L.spec_workspace_bytes_kv4.argtypes = [POINTER(spec_model_config), c_int32, c_int32, c_int32,
                                           c_int32]
    L.spec_workspace_bytes_kv4.restype = c_size_t
    L.spec_verify_kv4.argtypes = L.spec_verify_sampled.argtypes
    L.spec_workspace_bytes_w4.argtypes = L.spec_workspace_bytes_kv4.argtypes
    L.spec_workspace_bytes_w4.restype = c_size_t
    L.spec_verify_w4.argtypes = [POINTER(spec_model_config), POINTER(spec_weights_w4), c_void_p,
                                 *L.spec_verify_sampled.argtypes[2:]]
    w4 = POINTER(spec_w4)
    L.spec_w4_bytes.argtypes = [c_int32, c_int32]
    L.spec_w4_workspace_bytes.argtypes = [c_int32, c_int32, c_int32]
    L.spec_w4_product_bytes.argtypes = [c_int32] * 4
    L.spec_w4_pack.argtypes = [c_void_p, c_int64, c_int32, c_int32, c_void_p, c_size_t, c_void_p]
    L.spec_w4_unpack.argtypes = [w4, c_void_p, c_int64, c_void_p]
    L.spec_w4_linear.argtypes = [w4, c_void_p, c_int64, c_int32, c_void_p, c_int64, c_int32, c_void_p,
                                 c_size_t, c_void_p]
    L.spec_w4_gate_up.argtypes = [w4, w4, c_void_p, c_int64, c_int32, c_void_p, c_int64, c_void_p,
                                  c_size_t, c_void_p]
    L.spec_beam_workspace_bytes.argtypes = [c_int32] * 4
    L.spec_beam_select.argtypes = [c_void_p, c_int64, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p,
                                   c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                   c_void_p]
    L.spec_kv_reorder.argtypes = [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    L.spec_kv4_reorder_bytes.argtypes = [c_void_p, c_int32, c_int32, c_int32]
    L.spec_kv4_reorder.argtypes = [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_size_t, c_void_p]
    for name in ("spec_w4_bytes", "spec_w4_workspace_bytes", "spec_w4_product_bytes", "spec_beam_workspace_bytes",
                 "spec_kv4_reorder_bytes"):
        getattr(L, name).restype = c_size_t
    for name in ("spec_w4_pack", "spec_w4_unpack", "spec_w4_linear", "spec_w4_gate_up", "spec_beam_select",
                 "spec_kv_reorder", "spec_kv4_reorder", "spec_verify_kv4", "spec_verify_w4",
                 "spec_kv_alloc", "spec_kv_free", "spec_kv_sample_layout", "spec_verify",
                 "spec_kv_commit", "spec_profile_begin", "spec_profile_end", "spec_kv_pack",
                 "spec_kv_unpack", "spec_cost_model_create", "spec_cost_model_free",
                 "spec_cost_model_stats", "spec_select_draft_count", "spec_verify_sampled",
                 "spec_verify_noalloc", "spec_gemm_plan", "spec_kv4_alloc", "spec_kv4_free",
                 "spec_kv4_map", "spec_kv4_step_begin", "spec_kv4_step_free", "spec_kv4_append",
                 "spec_kv4_read", "spec_kv4_attend", "spec_kv4_commit"):
        getattr(L, name).restype = c_int32
    _lib = L
    return L


def _check(rc):
    if rc != 0:
        raise SpecError(rc, lib().spec_last_error().decode())


def _pointer(arr, kind):
    """A pointer to a contiguous array's data that keeps the array.  (The array's own
    ctypes.data_as leaves a reference cycle; a few per call bring Python's full collection,
    25 ms with torch loaded, into every 40th verify step or so.)"""
    p = POINTER(kind)(kind.from_address(arr.ctypes.data))
    p.arr = arr
    return p


def _i32(a):
    arr = np.ascontiguousarray(a, dtype=np.int32)
    return arr, _pointer(arr, c_int32)


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:      # the raw handle: a Stream object takes 3 us to make
        return c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return c_void_p(stream.cuda_stream)


def make_config(cfg) -> spec_model_config:
    return spec_model_config(cfg.n_layers, cfg.hidden, cfg.n_heads, cfg.n_kv_heads, cfg.head_dim,
                             cfg.ffn, cfg.vocab, float(cfg.rope_theta), float(cfg.rms_eps))


class Weights:
    """Device bf16 weights plus the spec_weights struct pointing at them."""

    LAYER_FIELDS = ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")

    def __init__(self, W):
        self.W = W
        for t in [W["tok_embed"], W["final_norm"], W["lm_head"]] + \
                [lw[k] for lw in W["layers"] for k in self.LAYER_FIELDS]:
            if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
                raise ValueError("weights must be contiguous bf16 device tensors")
        n = len(W["layers"])
        self._arrays = {}
        for k in self.LAYER_FIELDS:
            arr = (c_void_p * n)(*[lw[k].data_ptr() for lw in W["layers"]])
            self._arrays[k] = arr
        self.struct = spec_weights(W["tok_embed"].data_ptr(), W["final_norm"].data_ptr(),
                                   W["lm_head"].data_ptr(),
                                   *[ctypes.cast(self._arrays[k], POINTER(c_void_p))
                                     for k in self.LAYER_FIELDS])


def spec_kv_bytes(cfg, capacity) -> int:
    c = make_config(cfg)
    arr, p = _i32(capacity)
    return int(lib().spec_kv_bytes(ctypes.byref(c), len(arr), p))


class KVPool:
    """A KV pool over a torch-owned device buffer (spec_kv_alloc)."""

    def __init__(self, cfg, capacity, device="cuda"):
        self.cfg = cfg
        self.ccfg = make_config(cfg)
        self.capacity = [int(c) for c in capacity]
        nbytes = spec_kv_bytes(cfg, self.capacity)
        if nbytes == 0:
            raise SpecError(-1, "invalid KV pool request")
        self.buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.index = self.buf.get_device()
        self.handle = spec_kv_alloc(cfg, self.capacity, self.buf)

    def sample_view(self, sample):
        """(K, V) views of one sample, each [n_layers, n_kv_heads, capacity, head_dim]."""
        off, cap = spec_kv_sample_layout(self.handle, sample)
        c = self.cfg
        n = c.n_layers * 2 * c.n_kv_heads * cap * c.head_dim
        blk = self.buf[off:off + 2 * n].view(torch.bfloat16)
        blk = blk.view(c.n_layers, 2, c.n_kv_heads, cap, c.head_dim)
        return blk[:, 0], blk[:, 1]

    def close(self):
        if self.handle is not None:
            spec_kv_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def spec_kv_alloc(cfg, capacity, buf):
    c = make_config(cfg)
    arr, p = _i32(capacity)
    h = c_void_p()
    _check(lib().spec_kv_alloc(ctypes.byref(c), len(arr), p, c_void_p(buf.data_ptr()),
                               buf.numel() * buf.element_size(), ctypes.byref(h)))
    return h


def spec_kv_free(handle):
    _check(lib().spec_kv_free(handle))


def spec_kv_sample_layout(handle, sample):
    off, cap = c_int64(), c_int32()
    _check(lib().spec_kv_sample_layout(handle, sample, ctypes.byref(off), ctypes.byref(cap)))
    return off.value, cap.value


def spec_workspace_bytes(cfg, max_batch, max_tokens) -> int:
    c = make_config(cfg)
    return int(lib().spec_workspace_bytes(ctypes.byref(c), max_batch, max_tokens))


def spec_verify(cfg, weights: Weights, kv: KVPool, sample_ids, tree_offsets, tree_tokens,
                tree_parents, seq_lens, workspace, accepted_len, next_token, accepted_nodes,
                debug=None, stream=None):
    """Enqueue one verify step.  Host arrays may be lists or numpy arrays;
    workspace and outputs are device tensors; ``debug`` is an optional dict
    with any of logits/argmax/depth/pos/anc device tensors."""
    c = make_config(cfg)
    ids, p_ids = _i32(sample_ids)
    offs, p_offs = _i32(tree_offsets)
    toks, p_toks = _i32(tree_tokens)
    pars, p_pars = _i32(tree_parents)
    lens, p_lens = _i32(seq_lens)
    dbg = None
    if debug:
        dbg = spec_debug(*[debug[k].data_ptr() if debug.get(k) is not None else None
                           for k in ("logits", "argmax", "depth", "pos", "anc")])
    _check(lib().spec_verify(ctypes.byref(c), ctypes.byref(weights.struct), kv.handle,
                             len(ids), p_ids, p_offs, p_toks, p_pars, p_lens,
                             _ptr(workspace), workspace.numel() * workspace.element_size(),
                             _stream(stream), _ptr(accepted_len), _ptr(next_token),
                             _ptr(accepted_nodes), ctypes.byref(dbg) if dbg else None))


def spec_verify_noalloc(cfg, weights: Weights, kv: KVPool, sample_ids, tree_offsets, tree_tokens,
                        tree_parents, seq_lens, accepted_len, next_token, accepted_nodes,
                        debug=None, stream=None):
    """spec_verify with the library's static device scratch as workspace."""
    c = make_config(cfg)
    ids, p_ids = _i32(sample_ids)
    offs, p_offs = _i32(tree_offsets)
    toks, p_toks = _i32(tree_tokens)
    pars, p_pars = _i32(tree_parents)
    lens, p_lens = _i32(seq_lens)
    dbg = None
    if debug:
        dbg = spec_debug(*[debug[k].data_ptr() if debug.get(k) is not None else None
                           for k in ("logits", "argmax", "depth", "pos", "anc")])
    _check(lib().spec_verify_noalloc(ctypes.byref(c), ctypes.byref(weights.struct), kv.handle,
                                     len(ids), p_ids, p_offs, p_toks, p_pars, p_lens,
                                     _stream(stream), _ptr(accepted_len), _ptr(next_token),
                                     _ptr(accepted_nodes), ctypes.byref(dbg) if dbg else None))


def spec_workspace_bytes_sampled(cfg, max_batch, max_tokens) -> int:
    c = make_config(cfg)
    return int(lib().spec_workspace_bytes_sampled(ctypes.byref(c), max_batch, max_tokens))


def _sampling(cfg, n, temperature, eos_token, draft_probs, uniforms) -> spec_sampling:
    if temperature > 0:
        for t, cols, what in ((draft_probs, cfg.vocab, "draft_probs"), (uniforms, 2, "uniforms")):
            if (t is None or t.dtype != torch.float32 or not t.is_contiguous()
                    or tuple(t.shape) != (n, cols)):
                raise ValueError(f"{what} must be a contiguous float32 [{n}, {cols}] tensor")
    return spec_sampling(float(temperature), int(eos_token), _ptr(draft_probs), _ptr(uniforms))


def spec_verify_sampled(cfg, weights: Weights, kv: KVPool, sample_ids, tree_offsets, tree_tokens,
                        tree_parents, seq_lens, workspace, accepted_len, next_token,
                        accepted_nodes, temperature, eos_token=-1, draft_probs=None,
                        uniforms=None, debug=None, stream=None):
    """spec_verify with speculative-sampling acceptance at ``temperature`` (0:
    greedy) and end-of-sequence truncation.  draft_probs: device fp32
    [N][vocab]; uniforms: device fp32 [N][2]."""
    c = make_config(cfg)
    ids, p_ids = _i32(sample_ids)
    offs, p_offs = _i32(tree_offsets)
    toks, p_toks = _i32(tree_tokens)
    pars, p_pars = _i32(tree_parents)
    lens, p_lens = _i32(seq_lens)
    samp = _sampling(cfg, int(offs[-1]), temperature, eos_token, draft_probs, uniforms)
    dbg = None
    if debug:
        dbg = spec_debug(*[debug[k].data_ptr() if debug.get(k) is not None else None
                           for k in ("logits", "argmax", "depth", "pos", "anc")])
    _check(lib().spec_verify_sampled(ctypes.byref(c), ctypes.byref(weights.struct), kv.handle,
                                     len(ids), p_ids, p_offs, p_toks, p_pars, p_lens,
                                     _ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream), ctypes.byref(samp), _ptr(accepted_len),
                                     _ptr(next_token), _ptr(accepted_nodes),
                                     ctypes.byref(dbg) if dbg else None))


def spec_kv_commit(kv: KVPool, sample_ids, seq_lens, accepted_len, accepted_nodes, new_seq_lens,
                   stream=None):
    ids, p_ids = _i32(sample_ids)
    lens, p_lens = _i32(seq_lens)
    _check(lib().spec_kv_commit(kv.handle, len(ids), p_ids, p_lens, _ptr(accepted_len),
                                _ptr(accepted_nodes), _ptr(new_seq_lens), _stream(stream)))


def spec_kv_transfer_bytes(kv: KVPool, tok_begin, tok_end) -> int:
    b, p_b = _i32(tok_begin)
    e, p_e = _i32(tok_end)
    return int(lib().spec_kv_transfer_bytes(kv.handle, len(b), p_b, p_e))


def spec_kv_pack(kv: KVPool, sample_ids, tok_begin, tok_end, buf, stream=None):
    """Copy token ranges of the given samples into the transfer buffer ``buf``
    (a device tensor of at least spec_kv_transfer_bytes bytes)."""
    ids, p_ids = _i32(sample_ids)
    b, p_b = _i32(tok_begin)
    e, p_e = _i32(tok_end)
    _check(lib().spec_kv_pack(kv.handle, len(ids), p_ids, p_b, p_e, _ptr(buf),
                              buf.numel() * buf.element_size(), _stream(stream)))


def spec_kv_unpack(kv: KVPool, sample_ids, tok_begin, tok_end, buf, stream=None):
    """Write a transfer buffer's runs into token ranges of this pool's samples."""
    ids, p_ids = _i32(sample_ids)
    b, p_b = _i32(tok_begin)
    e, p_e = _i32(tok_end)
    _check(lib().spec_kv_unpack(kv.handle, len(ids), p_ids, p_b, p_e, _ptr(buf),
                                buf.numel() * buf.element_size(), _stream(stream)))


def spec_kv4_page_bytes(cfg) -> int:
    c = make_config(cfg)
    return int(lib().spec_kv4_page_bytes(ctypes.byref(c)))


def spec_kv4_bytes(cfg, n_samples, n_pages) -> int:
    c = make_config(cfg)
    return int(lib().spec_kv4_bytes(ctypes.byref(c), n_samples, n_pages))


def spec_kv4_step_bytes(cfg, max_batch, max_rows, max_pages) -> int:
    c = make_config(cfg)
    return int(lib().spec_kv4_step_bytes(ctypes.byref(c), max_batch, max_rows, max_pages))


_NOTHING = contextlib.nullcontext()


def _on(index):
    """torch.cuda.device(index), which costs nothing when that is the current one."""
    return _NOTHING if torch.cuda.current_device() == index else torch.cuda.device(index)


class KV4Pool:
    """A 4-bit paged KV pool over a torch-owned device buffer (spec_kv4_alloc)."""

    def __init__(self, cfg, n_samples, n_pages, buf=None, device="cuda"):
        """buf: a contiguous uint8 device tensor of at least spec_kv4_bytes bytes (allocated
        on ``device`` when None)."""
        self.handle = None
        self.cfg = cfg
        self.n_samples, self.n_pages = int(n_samples), int(n_pages)
        self.pages = {}
        nbytes = spec_kv4_bytes(cfg, self.n_samples, self.n_pages)
        if nbytes == 0:
            raise SpecError(-1, "invalid KV pool request")
        if buf is None:
            if torch.device(device).type != "cuda":
                raise ValueError(f"a KV pool lies in device memory, not on {device!r}")
            buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        elif buf.dtype != torch.uint8 or not buf.is_cuda or not buf.is_contiguous():
            raise ValueError("buf must be a contiguous uint8 device tensor")
        self.buf = buf
        self.index = buf.get_device()
        c = make_config(cfg)
        h = c_void_p()
        with _on(self.index):
            _check(lib().spec_kv4_alloc(ctypes.byref(c), self.n_samples, self.n_pages,
                                        c_void_p(buf.data_ptr()), buf.numel(), ctypes.byref(h)))
        self.handle = h

    def map(self, sample, pages):
        """Set the pages of one sample (spec_kv4_map)."""
        arr, p = _i32(pages)
        _check(lib().spec_kv4_map(self.handle, int(sample), len(arr), p))
        self.pages[int(sample)] = arr.tolist()

    def close(self):
        if self.handle is not None:
            h, self.handle = self.handle, None
            _check(lib().spec_kv4_free(h))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _kv4_arrays(sample_ids, row_offsets, seq_lens, **per_row):
    """The int32 arrays and pointers of a step's host arguments, which the library reads by
    the lengths of sample_ids and the last offset."""
    ids, offs, lens = (_i32(x) for x in (sample_ids, row_offsets, seq_lens))
    if len(offs[0]) != len(ids[0]) + 1 or len(lens[0]) != len(ids[0]):
        raise ValueError("row_offsets must have one entry more than sample_ids, seq_lens as many")
    rows = {name: (None, None) if x is None else _i32(x) for name, x in per_row.items()}
    for name, (arr, _) in rows.items():
        if len(ids[0]) and arr is not None and len(arr) != int(offs[0][-1]):
            raise ValueError(f"{name} must have one entry per row")
    return (ids, offs, lens, *rows.values())


def _kv4_stream(pool, stream):
    if stream is not None and stream.device.index != pool.index:
        raise ValueError(f"the stream is on {stream.device}, the pool on device {pool.index}")


def _kv4_workspace(pool, workspace):
    if (workspace.dtype != torch.uint8 or workspace.device != pool.buf.device
            or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor on the pool's device")


class KV4Step:
    """The plan of one step over a KV4Pool (spec_kv4_step_begin).

    parents: the trees' parents, or None for runs.  workspace: a uint8 tensor on the pool's
    device of at least spec_kv4_step_bytes bytes (allocated when None).  The step's launches
    go to streams of the pool's device."""

    def __init__(self, pool: KV4Pool, sample_ids, row_offsets, parents, seq_lens, workspace=None,
                 stream=None):
        self.handle = None
        self.pool = pool
        (ids, p_ids), (offs, p_offs), (lens, p_lens), (pars, p_pars) = _kv4_arrays(
            sample_ids, row_offsets, seq_lens, parents=parents)
        _kv4_stream(pool, stream)
        self.n_rows = int(offs[-1])
        self._made_on = None                 # the stream of a workspace of the step's own
        if workspace is None:
            pages = int(((lens.astype(np.int64) + np.diff(offs) + SPEC_KV4_PAGE - 1)
                         // SPEC_KV4_PAGE).sum())
            nbytes = spec_kv4_step_bytes(pool.cfg, len(ids), self.n_rows, max(pages, 1))
            # of that stream, where nothing before it can still use the memory
            with torch.cuda.stream(stream):
                workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=pool.buf.device)
            self._made_on = (torch._C._cuda_getCurrentRawStream(pool.index) if stream is None
                             else stream.cuda_stream)
        else:
            _kv4_workspace(pool, workspace)
        self.workspace = workspace
        h = c_void_p()
        with _on(pool.index):
            _check(lib().spec_kv4_step_begin(pool.handle, len(ids), p_ids, p_offs, p_pars, p_lens,
                                             _ptr(workspace),
                                             workspace.numel() * workspace.element_size(),
                                             self._on_stream(stream), ctypes.byref(h)))
        self.handle = h

    def _on_stream(self, stream):
        """The stream's handle.  A workspace of the step's own is not given away before that
        stream has passed its use."""
        if self.pool.handle is None:
            raise ValueError("the step's pool is closed")
        if stream is None:
            s = torch._C._cuda_getCurrentRawStream(self.pool.index)
        else:
            _kv4_stream(self.pool, stream)
            s = stream.cuda_stream
        if self._made_on is not None and s != self._made_on:
            self.workspace.record_stream(torch.cuda.current_stream() if stream is None else stream)
        return s

    def close(self):
        if self.handle is not None:
            h, self.handle = self.handle, None
            _check(lib().spec_kv4_step_free(h))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _kv4_rows(step, t, heads, what):
    """Row stride of a bf16 device tensor [rows, heads, head_dim] or [rows, heads * head_dim] whose
    rows are contiguous."""
    d = step.pool.cfg.head_dim
    if t.shape == (step.n_rows, heads, d) and t.is_contiguous() and t.dtype is torch.bfloat16 \
            and t.get_device() == step.pool.index:
        return heads * d
    flat = t.dim() == 2 and t.shape[1] == heads * d and t.stride(1) == 1
    split = (t.dim() == 3 and tuple(t.shape[1:]) == (heads, d) and t.stride(2) == 1
             and (heads == 1 or t.stride(1) == d))
    if (t.dtype != torch.bfloat16 or t.device != step.pool.buf.device or t.shape[0] != step.n_rows
            or not (flat or split)):
        raise ValueError(f"{what} must be a bfloat16 [{step.n_rows}, {heads}, {d}] tensor on the "
                         "pool's device with contiguous rows")
    return t.stride(0) if step.n_rows > 1 else heads * d


def _kv4_tensors(pool, dtype, **tensors):
    """Each name=(tensor, numbers) must be a contiguous tensor of that type on the pool's device
    that holds that many."""
    for name, (t, n) in tensors.items():
        if (t.dtype != dtype or t.device != pool.buf.device or not t.is_contiguous()
                or t.numel() < n):
            kind = str(dtype).split(".")[-1]
            raise ValueError(f"{name} must be a contiguous {kind} tensor of {n} on the pool's device")


def spec_kv4_append(step: KV4Step, layer, k, v, rotate=True, stream=None):
    """Write the rows' K and V ([rows, kv heads, head_dim], rows may be strided) into the cache,
    rotating k by position unless it has been."""
    if torch.cuda.current_device() != step.pool.index:
        with torch.cuda.device(step.pool.index):
            return spec_kv4_append(step, layer, k, v, rotate, stream)
    n = step.pool.cfg.n_kv_heads
    ks, vs = _kv4_rows(step, k, n, "k"), _kv4_rows(step, v, n, "v")
    rc = lib().spec_kv4_append(step.handle, int(layer), k.data_ptr(), ks, v.data_ptr(), vs, bool(rotate),
                               step._on_stream(stream))
    if rc:
        _check(rc)


def spec_kv4_read(step: KV4Step, layer, k, v, stream=None):
    """Write what the cache holds for the step's rows into k and v (as in spec_kv4_append)."""
    if torch.cuda.current_device() != step.pool.index:
        with torch.cuda.device(step.pool.index):
            return spec_kv4_read(step, layer, k, v, stream)
    n = step.pool.cfg.n_kv_heads
    ks, vs = _kv4_rows(step, k, n, "k"), _kv4_rows(step, v, n, "v")
    rc = lib().spec_kv4_read(step.handle, int(layer), k.data_ptr(), ks, v.data_ptr(), vs,
                             step._on_stream(stream))
    if rc:
        _check(rc)


def spec_kv4_attend(step: KV4Step, layer, q, out, stream=None):
    """Attention of the step's rows: q [rows, heads, head_dim] (rows may be strided), rotated;
    out [rows, heads * head_dim], contiguous."""
    if torch.cuda.current_device() != step.pool.index:
        with torch.cuda.device(step.pool.index):
            return spec_kv4_attend(step, layer, q, out, stream)
    n = step.pool.cfg.n_heads
    qs = _kv4_rows(step, q, n, "q")
    _kv4_rows(step, out, n, "out")
    if not out.is_contiguous():
        raise ValueError("out must be contiguous")
    rc = lib().spec_kv4_attend(step.handle, int(layer), q.data_ptr(), qs, out.data_ptr(),
                               step._on_stream(stream))
    if rc:
        _check(rc)


def spec_workspace_bytes_kv4(cfg, max_batch, max_tokens, max_pages, sampled=False) -> int:
    c = make_config(cfg)
    return int(lib().spec_workspace_bytes_kv4(ctypes.byref(c), max_batch, max_tokens, max_pages,
                                              int(sampled)))


def spec_verify_kv4(cfg, weights: Weights, pool: KV4Pool, sample_ids, tree_offsets, tree_tokens,
                    tree_parents, seq_lens, workspace, accepted_len, next_token, accepted_nodes,
                    temperature=0.0, eos_token=-1, draft_probs=None, uniforms=None, debug=None,
                    stream=None):
    """spec_verify (or, with a temperature or an EOS token, spec_verify_sampled) over a 4-bit
    pool."""
    _verify_pool(lib().spec_verify_kv4, (ctypes.byref(weights.struct), pool.handle), cfg, pool, sample_ids,
                 tree_offsets, tree_tokens, tree_parents, seq_lens, workspace, accepted_len, next_token,
                 accepted_nodes, temperature, eos_token, draft_probs, uniforms, debug, stream)


def _verify_pool(call, handles, cfg, pool, sample_ids, tree_offsets, tree_tokens, tree_parents, seq_lens,
                 workspace, accepted_len, next_token, accepted_nodes, temperature, eos_token, draft_probs,
                 uniforms, debug, stream):
    """call, one of the verify steps, after checks of every array and tensor that it reads."""
    c = make_config(cfg)
    (ids, p_ids), (offs, p_offs), (lens, p_lens), (_, p_toks), (_, p_pars) = _kv4_arrays(
        sample_ids, tree_offsets, seq_lens, tree_tokens=tree_tokens, tree_parents=tree_parents)
    n = int(offs[-1])
    _kv4_stream(pool, stream)
    _kv4_workspace(pool, workspace)
    samp = _sampling(cfg, n, temperature, eos_token, draft_probs, uniforms)
    if temperature > 0:
        _kv4_tensors(pool, torch.float32, draft_probs=(draft_probs, n * cfg.vocab), uniforms=(uniforms, 2 * n))
    _kv4_tensors(pool, torch.int32, accepted_len=(accepted_len, len(ids)), next_token=(next_token, len(ids)),
                 accepted_nodes=(accepted_nodes, len(ids) * SPEC_MAX_TREE))
    dbg = None
    if debug:
        for name, dtype, width in (("logits", torch.float32, cfg.vocab), ("argmax", torch.int32, 1),
                                   ("depth", torch.int32, 1), ("pos", torch.int32, 1),
                                   ("anc", torch.int64, SPEC_ANC_WORDS)):
            if debug.get(name) is not None:
                _kv4_tensors(pool, dtype, **{name: (debug[name], n * width)})
        dbg = spec_debug(*[debug[k].data_ptr() if debug.get(k) is not None else None
                           for k in ("logits", "argmax", "depth", "pos", "anc")])
    with _on(pool.index):
        _check(call(ctypes.byref(c), *handles, len(ids), p_ids, p_offs, p_toks, p_pars, p_lens, _ptr(workspace),
                    workspace.numel() * workspace.element_size(), _stream(stream), ctypes.byref(samp),
                    _ptr(accepted_len), _ptr(next_token), _ptr(accepted_nodes),
                    ctypes.byref(dbg) if dbg else None))


def spec_kv4_commit(pool: KV4Pool, sample_ids, seq_lens, accepted_len, accepted_nodes, new_seq_lens,
                    stream=None):
    ids, p_ids = _i32(sample_ids)
    lens, p_lens = _i32(seq_lens)
    if len(lens) != len(ids):
        raise ValueError("seq_lens must have as many entries as sample_ids")
    _kv4_stream(pool, stream)
    _kv4_tensors(pool, torch.int32, accepted_len=(accepted_len, len(ids)), new_seq_lens=(new_seq_lens, len(ids)),
                 accepted_nodes=(accepted_nodes, len(ids) * SPEC_MAX_TREE))
    with _on(pool.index):
        _check(lib().spec_kv4_commit(pool.handle, len(ids), p_ids, p_lens, _ptr(accepted_len),
                                     _ptr(accepted_nodes), _ptr(new_seq_lens), _stream(stream)))


# ---- products with weights in 4 bits ----

@functools.lru_cache(maxsize=4096)
def spec_w4_bytes(rows, cols) -> int:
    return int(lib().spec_w4_bytes(rows, cols))


def spec_w4_workspace_bytes(rows, cols, max_n) -> int:
    return int(lib().spec_w4_workspace_bytes(rows, cols, max_n))


def spec_w4_product_bytes(rows, cols, n, pair=False) -> int:
    return int(lib().spec_w4_product_bytes(rows, cols, n, int(bool(pair))))


def _device_rows(t, dtype, rows, cols, what, index=None):
    """Row stride of a device tensor [rows, cols] whose rows are contiguous."""
    shape = t.shape
    if t.dtype is dtype and t.is_cuda and len(shape) == 2 and shape[1] == cols and not cols & 7 \
            and t.get_device() == index and (rows is None or shape[0] == rows) and t.is_contiguous():
        return cols
    if t.dtype is not dtype or not t.is_cuda or t.dim() != 2 or t.shape[1] != cols \
            or (rows is not None and t.shape[0] != rows) or (t.stride(1) != 1 and cols > 1) \
            or (index is not None and t.get_device() != index):
        kind = str(dtype).split(".")[-1]
        where = "a device" if index is None or index < 0 else f"cuda:{index}"
        raise ValueError(f"{what} must be a {kind} [{'n' if rows is None else rows}, {cols}] tensor on {where} with "
                         "contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else max(cols, (cols + 7) // 8 * 8)


def _device_stream(index, stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index)
    if stream.device.index != index:
        raise ValueError(f"the stream is on {stream.device}, the tensors on device {index}")
    return stream.cuda_stream


def _device_workspace(workspace, index):
    """(pointer, bytes) of a workspace tensor."""
    if workspace.dtype is not torch.uint8 or workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the tensors' device")
    return workspace.data_ptr(), workspace.numel()


def _made_workspace(nbytes, index, stream):
    """A workspace that lives until `stream` has passed what is launched on it next."""
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", index))


def spec_w4_pack(w, data, stream=None):
    """Quantise w (bf16 [rows, cols], rows may be strided) into data (uint8, spec_w4_bytes)."""
    rows, cols = w.shape if w.dim() == 2 else (0, 0)
    index = w.get_device()
    stride = _device_rows(w, torch.bfloat16, rows, cols, "w", index)
    p, n = _device_workspace(data, index)
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return spec_w4_pack(w, data, stream)
    rc = lib().spec_w4_pack(w.data_ptr(), stride, rows, cols, p, n, _device_stream(index, stream))
    if rc:
        _check(rc)


def spec_w4_unpack(data, w, stream=None):
    """Write what data (of spec_w4_pack) stands for into w (bf16 [rows, cols])."""
    rows, cols = w.shape if w.dim() == 2 else (0, 0)
    index = w.get_device()
    stride = _device_rows(w, torch.bfloat16, rows, cols, "w", index)
    p, n = _device_workspace(data, index)
    if n < spec_w4_bytes(rows, cols):
        raise ValueError(f"data holds {n} bytes, a matrix of {rows} x {cols} {spec_w4_bytes(rows, cols)}")
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return spec_w4_unpack(data, w, stream)
    rc = lib().spec_w4_unpack(spec_w4(p, rows, cols), w.data_ptr(), stride, _device_stream(index, stream))
    if rc:
        _check(rc)


class W4Matrix:
    """A weight matrix [rows, cols] in 4 bits, quantised from a bf16 device tensor."""

    def __init__(self, w, stream=None):
        if w.dim() != 2 or not w.is_cuda:
            raise ValueError("a weight matrix is a bfloat16 [rows, cols] device tensor")
        self.rows, self.cols = w.shape
        self.index = w.get_device()
        nbytes = spec_w4_bytes(self.rows, self.cols)
        if nbytes == 0:
            raise SpecError(-6, f"a matrix of {self.rows} x {self.cols}: columns must be a multiple of 32")
        self.data = _made_workspace(nbytes, self.index, stream)
        spec_w4_pack(w, self.data, stream)
        self.struct = spec_w4(self.data.data_ptr(), self.rows, self.cols)
        self.needs = {}                      # workspace bytes by rows of x, alone and of a pair

    def unpack(self, out=None, stream=None):
        """What the matrix stands for, as bf16."""
        if out is None:
            with torch.cuda.stream(stream):
                out = torch.empty(self.rows, self.cols, dtype=torch.bfloat16, device=self.data.device)
        elif out.shape != (self.rows, self.cols):
            raise ValueError(f"out must have the matrix's shape, {self.rows} x {self.cols}")
        spec_w4_unpack(self.data, out, stream)
        return out


class W4Weights:
    """A model's weights with its matrices in 4 bits, quantised from those that Weights takes
    (W["layers"] may be an iterator, so that a layer's bf16 matrices need not outlive it)."""

    MATRICES = ("wqkv", "wo", "w_gate", "w_up", "w_down")

    def __init__(self, W, stream=None):
        self.lm_head = W4Matrix(W["lm_head"], stream)
        self.index = self.lm_head.index
        self.tok_embed, self.final_norm = W["tok_embed"], W["final_norm"]
        self.norms, self.matrices = {"attn_norm": [], "ffn_norm": []}, {k: [] for k in self.MATRICES}
        with torch.cuda.stream(stream):
            for lw in W["layers"]:
                for k, rows in self.norms.items():
                    rows.append(lw[k])
                for k, layers in self.matrices.items():
                    w = torch.cat([lw["wq"], lw["wk"], lw["wv"]]) if k == "wqkv" else lw[k]
                    layers.append(W4Matrix(w, stream))
                    if layers[-1].index != self.index:
                        raise ValueError(f"{k} of layer {len(layers) - 1} is on another device than the head")
        n, gains = len(self.norms["attn_norm"]), [self.final_norm, *self.norms["attn_norm"], *self.norms["ffn_norm"]]
        vocab, hidden = self.tok_embed.shape
        for t in (self.tok_embed, *gains):
            if t.dtype != torch.bfloat16 or t.get_device() != self.index or not t.is_contiguous():
                raise ValueError("norm gains and the embedding must be contiguous bf16 tensors on the matrices' device")
        if any(t.shape != (hidden,) for t in gains):
            raise ValueError(f"norm gains must have the embedding's {hidden} values")
        self.shape = (n, hidden, vocab)
        self._arrays = {k: (c_void_p * n)(*[t.data_ptr() for t in rows]) for k, rows in self.norms.items()}
        self._arrays |= {k: (spec_w4 * n)(*[m.struct for m in layers]) for k, layers in self.matrices.items()}
        a = {k: ctypes.cast(v, POINTER(v._type_)) for k, v in self._arrays.items()}
        self.struct = spec_weights_w4(self.tok_embed.data_ptr(), self.final_norm.data_ptr(), self.lm_head.struct,
                                      a["attn_norm"], a["wqkv"], a["wo"], a["ffn_norm"], a["w_gate"], a["w_up"],
                                      a["w_down"])


def spec_workspace_bytes_w4(cfg, max_batch, max_tokens, max_pages=0, sampled=False) -> int:
    c = make_config(cfg)
    return int(lib().spec_workspace_bytes_w4(ctypes.byref(c), max_batch, max_tokens, max_pages, int(bool(sampled))))


def spec_verify_w4(cfg, weights: W4Weights, pool, sample_ids, tree_offsets, tree_tokens, tree_parents,
                   seq_lens, workspace, accepted_len, next_token, accepted_nodes, temperature=0.0, eos_token=-1,
                   draft_probs=None, uniforms=None, debug=None, stream=None):
    """spec_verify (or, with a temperature or an EOS token, spec_verify_sampled) with weights in 4
    bits, over a KVPool or a KV4Pool."""
    if weights.index != pool.index:
        raise ValueError(f"the weights are on device {weights.index}, the pool on device {pool.index}")
    if weights.shape != (cfg.n_layers, cfg.hidden, cfg.vocab):
        raise ValueError("the weights are of another shape than the model's")
    kv, kv4 = (None, pool.handle) if isinstance(pool, KV4Pool) else (pool.handle, None)
    _verify_pool(lib().spec_verify_w4, (ctypes.byref(weights.struct), kv, kv4), cfg, pool, sample_ids, tree_offsets,
                 tree_tokens, tree_parents, seq_lens, workspace, accepted_len, next_token, accepted_nodes,
                 temperature, eos_token, draft_probs, uniforms, debug, stream)


def _w4_workspace(m, n, pair, stream):
    """A workspace that a product needs, the caller's to hold until it is launched, or None."""
    nbytes = m.needs.get((n, pair))
    if nbytes is None:
        nbytes = m.needs[n, pair] = lib().spec_w4_product_bytes(m.rows, m.cols, n, pair)
    return _made_workspace(nbytes, m.index, stream) if nbytes else None


def spec_w4_linear(m: W4Matrix, x, out, add=False, workspace=None, stream=None):
    """out = x W^T: x bf16 [n, cols] (rows may be strided), out bf16 or float32 [n, rows]; add: float32
    out += x W^T.  workspace: a uint8 tensor of spec_w4_workspace_bytes (allocated when None)."""
    index = m.index
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return spec_w4_linear(m, x, out, add, workspace, stream)
    xs = _device_rows(x, torch.bfloat16, None, m.cols, "x", index)
    n = len(x)
    kind = SPEC_W4_ADD if add else SPEC_W4_BF16 if out.dtype is torch.bfloat16 else SPEC_W4_F32
    os = _device_rows(out, torch.float32 if kind else torch.bfloat16, n, m.rows, "out", index)
    if n == 0:
        return
    if workspace is None:
        workspace = _w4_workspace(m, n, 0, stream)
    p, nbytes = (None, 0) if workspace is None else _device_workspace(workspace, index)
    rc = lib().spec_w4_linear(m.struct, x.data_ptr(), xs, n, out.data_ptr(), os, kind, p, nbytes,
                              _device_stream(index, stream))
    if rc:
        _check(rc)


def spec_w4_gate_up(gate: W4Matrix, up: W4Matrix, x, out, workspace=None, stream=None):
    """out = silu(x Wg^T) * (x Wu^T), bf16 [n, rows]; the rest as in spec_w4_linear."""
    index = gate.index
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return spec_w4_gate_up(gate, up, x, out, workspace, stream)
    if up.index != index:
        raise ValueError("gate and up are on different devices")
    xs = _device_rows(x, torch.bfloat16, None, gate.cols, "x", index)
    n = len(x)
    os = _device_rows(out, torch.bfloat16, n, gate.rows, "out", index)
    if n == 0:
        return
    if workspace is None:
        workspace = _w4_workspace(gate, n, 1, stream)
    p, nbytes = (None, 0) if workspace is None else _device_workspace(workspace, index)
    rc = lib().spec_w4_gate_up(gate.struct, up.struct, x.data_ptr(), xs, n, out.data_ptr(), os, p, nbytes,
                               _device_stream(index, stream))
    if rc:
        _check(rc)


# ---- the choice of beams, and the cache rows that follow ----

def spec_beam_workspace_bytes(groups, width, vocab, k) -> int:
    return int(lib().spec_beam_workspace_bytes(groups, width, vocab, k))


def _beam_tensor(t, dtype, shape, index, what):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != index:
        kind = str(dtype).split(".")[-1]
        raise ValueError(f"{what} must be a contiguous {kind} tensor of {tuple(shape)} on the logits' device")
    return t.data_ptr()


def spec_beam_select(logits, scores, parents, tokens, new_scores, last_tokens=None, eos_token=-1, workspace=None,
                     stream=None):
    """The k best continuations of every group's beams.  logits float32 or bfloat16
    [groups, width, vocab] (rows may be strided, evenly); scores float32 and last_tokens int32
    [groups, width]; parents, tokens int32 and new_scores float32 [groups, k] are written."""
    if logits.dtype not in (torch.float32, torch.bfloat16) or not logits.is_cuda or logits.dim() != 3 \
            or parents.dim() != 2:
        raise ValueError("logits must be a float32 or bfloat16 [groups, width, vocab] device tensor, parents [groups, k]")
    groups, width, vocab = logits.shape
    index = logits.get_device()
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return spec_beam_select(logits, scores, parents, tokens, new_scores, last_tokens, eos_token, workspace,
                                    stream)
    by_group, by_row, by_token = logits.stride()
    row = by_row if width > 1 else by_group if groups > 1 else vocab
    if (by_token != 1 and vocab > 1) or (width > 1 and groups > 1 and by_group != width * by_row):
        raise ValueError("logits must have contiguous rows at one stride")
    k = parents.shape[1]
    beams, kept = torch.Size((groups, width)), torch.Size((groups, k))
    i32, f32 = torch.int32, torch.float32
    pointers = (_beam_tensor(scores, f32, beams, index, "scores"),
                None if last_tokens is None else _beam_tensor(last_tokens, i32, beams, index, "last_tokens"),
                int(eos_token), k, _beam_tensor(parents, i32, kept, index, "parents"),
                _beam_tensor(tokens, i32, kept, index, "tokens"),
                _beam_tensor(new_scores, f32, kept, index, "new_scores"))
    if workspace is None:
        workspace = _made_workspace(max(256, lib().spec_beam_workspace_bytes(groups, width, vocab, k)), index, stream)
    p, nbytes = _device_workspace(workspace, index)
    rc = lib().spec_beam_select(logits.data_ptr(), row, logits.dtype is torch.bfloat16, groups, width, vocab, *pointers,
                                p, nbytes, _device_stream(index, stream))
    if rc:
        _check(rc)


def _reorder_arrays(pool_index, sample_ids, begin, end, parents):
    """int32 arrays of a reorder call's host arguments."""
    ids, b, e = (np.ascontiguousarray(x, dtype=np.int32) for x in (sample_ids, begin, end))
    if ids.ndim != 2:
        raise ValueError("sample_ids must be [groups, width]")
    if b.shape != ids.shape[:1] or e.shape != b.shape:
        raise ValueError("begin and end must have one entry per group")
    if parents.dtype is not torch.int32 or parents.shape != ids.shape or not parents.is_contiguous() \
            or parents.get_device() != pool_index:
        raise ValueError(f"parents must be a contiguous int32 tensor of {ids.shape} on the pool's device")
    return ids, b, e


def spec_kv_reorder(pool: KVPool, sample_ids, begin, end, parents, stream=None):
    """Beam j of group g (sample sample_ids[g][j]) takes what beam parents[g][j] holds at positions
    [begin[g], end[g])."""
    index = pool.buf.get_device()
    ids, b, e = _reorder_arrays(index, sample_ids, begin, end, parents)
    if pool.handle is None:
        raise ValueError("the pool is closed")
    with _on(index):
        rc = lib().spec_kv_reorder(pool.handle, *ids.shape, ids.ctypes.data, b.ctypes.data, e.ctypes.data,
                                   parents.data_ptr(), _device_stream(index, stream))
    if rc:
        _check(rc)


def spec_kv4_reorder_bytes(pool: KV4Pool, groups, width, max_pages) -> int:
    return int(lib().spec_kv4_reorder_bytes(pool.handle, groups, width, max_pages))


def spec_kv4_reorder(pool: KV4Pool, sample_ids, begin, end, parents, workspace=None, stream=None):
    """spec_kv_reorder for a 4-bit pool; workspace: a uint8 tensor of spec_kv4_reorder_bytes
    (allocated when None and needed)."""
    index = pool.index
    ids, b, e = _reorder_arrays(index, sample_ids, begin, end, parents)
    if pool.handle is None:
        raise ValueError("the pool is closed")
    p, nbytes = None, 0
    if workspace is not None:
        p, nbytes = _device_workspace(workspace, index)
    elif ids.size:
        pages = min((int(e.max()) - 1) // SPEC_KV4_PAGE - int(b.min()) // SPEC_KV4_PAGE + 1, pool.n_pages)
        nbytes = lib().spec_kv4_reorder_bytes(pool.handle, *ids.shape, max(1, pages))
        if nbytes:
            workspace = _made_workspace(nbytes, index, stream)
            p = workspace.data_ptr()
    with _on(index):
        rc = lib().spec_kv4_reorder(pool.handle, *ids.shape, ids.ctypes.data, b.ctypes.data, e.ctypes.data,
                                    parents.data_ptr(), p, nbytes, _device_stream(index, stream))
    if rc:
        _check(rc)


class CostModel:
    """The library's verification-cost predictor (spec_cost_model_*)."""

    def __init__(self, c0, c_seq, c_draft, c_tree, bucket_ratio=0.0):
        self.coeffs = spec_cost_coeffs(c0, c_seq, c_draft, c_tree, bucket_ratio)
        h = c_void_p()
        _check(lib().spec_cost_model_create(ctypes.byref(self.coeffs), ctypes.byref(h)))
        self.handle = h

    @classmethod
    def from_dict(cls, d, bucket_ratio=None):
        return cls(d["c0"], d["c_seq"], d["c_draft"], d["c_tree"],
                   d.get("bucket_ratio", 0.0) if bucket_ratio is None else bucket_ratio)

    def predict(self, n_seq, n_draft, tree_kv):
        t = lib().spec_cost_predict(self.handle, int(n_seq), int(n_draft), int(tree_kv))
        if t < 0:
            raise SpecError(-1, "negative feature")
        return t

    def stats(self):
        h, m = c_int64(), c_int64()
        _check(lib().spec_cost_model_stats(self.handle, ctypes.byref(h), ctypes.byref(m)))
        return h.value, m.value

    def close(self):
        if self.handle is not None:
            _check(lib().spec_cost_model_free(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def spec_select_draft_count(model: CostModel, seq_lens, tree_offsets, parents, weights, n_max,
                            patience=2):
    """Returns (n, selected [batch][n_max] int32 array, objective [n_max])."""
    lens, p_lens = _i32(seq_lens)
    offs, p_offs = _i32(tree_offsets)
    pars, p_pars = _i32(parents)
    w = np.ascontiguousarray(np.asarray(weights, dtype=np.float32))
    sel = np.empty((len(lens), n_max), dtype=np.int32)
    obj = np.empty(n_max, dtype=np.float64)
    n = c_int32()
    _check(lib().spec_select_draft_count(model.handle, len(lens), p_lens, p_offs, p_pars,
                                         _pointer(w, c_float), n_max, patience, ctypes.byref(n),
                                         _pointer(sel, c_int32), _pointer(obj, ctypes.c_double)))
    return n.value, sel, obj


def spec_profile_begin(kernel_class, max_launches):
    if isinstance(kernel_class, str):
        k = OPERATOR_CLASS[kernel_class] if kernel_class in OPERATOR_CLASS else KERNEL_CLASS[kernel_class]
    else:
        k = int(kernel_class)
    _check(lib().spec_profile_begin(k, max_launches))


def spec_profile_end():
    ms, n = c_float(), c_int32()
    _check(lib().spec_profile_end(ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def spec_gemm_plan(cfg, kernel_class, n_tokens):
    """(tile rows, tile columns, K splits) of a product ("gemm_qkv", "gemm_o", "gemm_gate_up",
    "gemm_down", "lm_head") of a verify step of n_tokens rows; (0, 16, 1) on the few-rows kernel."""
    c = make_config(cfg)
    rows, cols, splits = c_int32(), c_int32(), c_int32()
    _check(lib().spec_gemm_plan(ctypes.byref(c), KERNEL_CLASS[kernel_class], n_tokens,
                                ctypes.byref(rows), ctypes.byref(cols), ctypes.byref(splits)))
    return rows.value, cols.value, splits.value
