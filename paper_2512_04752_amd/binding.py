"""ctypes binding of libspecverify.so: the C entry points under the same
names, marshalling torch tensors, numpy arrays and Python lists into
pointers.  Every step of the verify computation runs in the library's HIP
kernels; PyTorch only provides device memory and the stream.
"""

from __future__ import annotations

import contextlib
import ctypes
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
           "spec_workspace_bytes_kv4", "spec_verify_kv4")
SPEC_KV4_PAGE = 64                # positions per page of the 4-bit pool
SPEC_NOALLOC_SCRATCH_BYTES = 320 << 20


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
    for name in ("spec_verify_kv4", "spec_kv_alloc", "spec_kv_free", "spec_kv_sample_layout", "spec_verify",
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
    arr = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
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
        _check(lib().spec_verify_kv4(ctypes.byref(c), ctypes.byref(weights.struct), pool.handle,
                                     len(ids), p_ids, p_offs, p_toks, p_pars, p_lens, _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream(stream),
                                     ctypes.byref(samp), _ptr(accepted_len), _ptr(next_token),
                                     _ptr(accepted_nodes), ctypes.byref(dbg) if dbg else None))


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
    if kernel_class == "transfer":
        k = TRANSFER_CLASS
    elif kernel_class == "kv4_append":
        k = KV4_APPEND_CLASS
    else:
        k = KERNEL_CLASS[kernel_class] if isinstance(kernel_class, str) else int(kernel_class)
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
