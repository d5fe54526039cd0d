"""Python binding of the block-hybrid attention C ABI (include/hybrid.h, and
include/hybrid_softmax.h for the softmax layers of a hybrid model).

Argument marshalling only: every function here forwards to the entry point of
``libhybrid.so`` with the same name.  Tensors are passed as device pointers
(``tensor.data_ptr()``); torch is used for device memory and streams and
nothing else.  There is no fallback: if the library is missing or fails to
load, every call raises.
"""
from __future__ import annotations

import ctypes
import os

from . import build as _build

HYBRID_OK = 0
HYBRID_ERR_INVALID_ARG = 1
HYBRID_ERR_UNSUPPORTED = 2
HYBRID_ERR_CUDA = 3
HYBRID_ERR_TIMEOUT = 4
HYBRID_ERR_DEVICE = 5

HYBRID_F32 = 0
HYBRID_BF16 = 1

EXPORTED = (
    "hybrid_state_bytes", "hybrid_state_init", "hybrid_feature_map", "hybrid_block_attn",
    "hybrid_block_attn_commit", "hybrid_block_attn_commit_logical", "hybrid_commit_block", "hybrid_commit_ragged",
    "hybrid_state_unpack",
    "hybrid_state_pack", "hybrid_train_workspace_bytes", "hybrid_train_forward", "hybrid_train_backward",
    "hybrid_debug_arm_wait_timeout", "hybrid_check", "hybrid_status_str",
    # the softmax layers of a hybrid model (include/hybrid_softmax.h)
    "hybrid_page_append", "hybrid_page_release", "hybrid_rope_freqs", "hybrid_qk_norm_rope",
    "hybrid_qk_norm_rope_cache", "hybrid_qk_norm_rope_workspace_bytes", "hybrid_qk_norm_rope_backward",
    "hybrid_paged_attn_workspace_bytes", "hybrid_paged_attn",
    "hybrid_qk_norm_rope_cache_quant", "hybrid_cache_dequant", "hybrid_paged_attn_quant_workspace_bytes",
    "hybrid_paged_attn_quant",
)

HYBRID_QUANT_TOKENS = 16      # tokens of a head that share a scale in an 8-bit cache

HYBRID_ROPE_NONE = 0
HYBRID_ROPE_LINEAR = 1
HYBRID_ROPE_NTK = 2
HYBRID_ROPE_YARN = 3


class hybrid_cfg(ctypes.Structure):
    _fields_ = [
        ("head_dim", ctypes.c_int),
        ("feat_dim", ctypes.c_int),
        ("n_q_heads", ctypes.c_int),
        ("n_kv_heads", ctypes.c_int),
        ("block_size", ctypes.c_int),
        ("io_dtype", ctypes.c_int),
    ]

    def __repr__(self):
        return (f"hybrid_cfg(d={self.head_dim}, F={self.feat_dim}, Hq={self.n_q_heads}, "
                f"Hkv={self.n_kv_heads}, B={self.block_size}, io_dtype={self.io_dtype})")


class hybrid_page_cfg(ctypes.Structure):
    _fields_ = [("page_size", ctypes.c_int), ("n_pages", ctypes.c_int), ("max_pages", ctypes.c_int)]

    def __repr__(self):
        return f"hybrid_page_cfg(page_size={self.page_size}, n_pages={self.n_pages}, max_pages={self.max_pages})"


class hybrid_rope_cfg(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int), ("scale", ctypes.c_float),
                ("eps", ctypes.c_float)]

    def __repr__(self):
        return (f"hybrid_rope_cfg(rot_dim={self.rot_dim}, interleaved={self.interleaved}, scale={self.scale}, "
                f"eps={self.eps})")


class hybrid_rope_scaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("orig_len", ctypes.c_double), ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double)]


class HybridError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {hybrid_status_str(status)}")
        self.status = status


_lib = None


def lib(path: str | None = None):
    """Load libhybrid.so (once).  Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or _build.LIB_PATH
    if not os.path.exists(path):
        raise ImportError(f"libhybrid.so not built ({path}); run __graft_entry__.build()")
    L = ctypes.CDLL(path)
    P = ctypes.c_void_p
    I = ctypes.c_int
    cfgp = ctypes.POINTER(hybrid_cfg)
    L.hybrid_state_bytes.argtypes = [cfgp]
    L.hybrid_state_bytes.restype = ctypes.c_size_t
    L.hybrid_state_init.argtypes = [cfgp, P, I, P]
    L.hybrid_feature_map.argtypes = [cfgp, P, I, I, P, P, P]
    L.hybrid_block_attn.argtypes = [cfgp, P, P, P, P, P, P, I, P, P]
    L.hybrid_block_attn_commit.argtypes = [cfgp, P, P, P, P, P, P, I, P, P]
    L.hybrid_block_attn_commit_logical.argtypes = [cfgp, P, P, P, P, P, P, P, I, P, P]
    L.hybrid_commit_block.argtypes = [cfgp, P, P, I, P, P, I, P]
    L.hybrid_commit_ragged.argtypes = [cfgp, P, P, ctypes.POINTER(ctypes.c_int), I, P, P, P]
    L.hybrid_state_unpack.argtypes = [cfgp, P, I, P, P, P]
    L.hybrid_state_pack.argtypes = [cfgp, P, P, P, I, P]
    S = ctypes.c_size_t
    L.hybrid_train_workspace_bytes.argtypes = [cfgp, I, I]
    L.hybrid_train_workspace_bytes.restype = S
    L.hybrid_train_forward.argtypes = [cfgp, P, P, P, P, P, I, I, P, P, S, P]
    L.hybrid_train_backward.argtypes = [cfgp, P, P, P, P, P, P, I, I, P, S, P, P, P]
    L.hybrid_debug_arm_wait_timeout.argtypes = [ctypes.c_ulonglong]
    L.hybrid_check.argtypes = [P]
    L.hybrid_status_str.argtypes = [I]
    L.hybrid_status_str.restype = ctypes.c_char_p
    pgp, ropep = ctypes.POINTER(hybrid_page_cfg), ctypes.POINTER(hybrid_rope_cfg)
    L.hybrid_page_append.argtypes = [pgp, I, P, P, P, P, P, P, P, I, P, P, P, P]
    L.hybrid_page_release.argtypes = [pgp, I, P, I, P, P, P, P, P, P]
    L.hybrid_rope_freqs.argtypes = [ctypes.POINTER(hybrid_rope_scaling), I, P, ctypes.POINTER(ctypes.c_float)]
    L.hybrid_qk_norm_rope.argtypes = [cfgp, ropep, P, S, P, S, I, P, P, P, P, P, P, P]
    L.hybrid_qk_norm_rope_cache.argtypes = [cfgp, ropep, pgp, P, S, P, S, P, S, I, P, P, P, P, P, P, P, P, P]
    L.hybrid_qk_norm_rope_workspace_bytes.argtypes = [cfgp, I]
    L.hybrid_qk_norm_rope_workspace_bytes.restype = S
    L.hybrid_qk_norm_rope_backward.argtypes = [cfgp, ropep, P, S, P, S, P, P, I, P, P, P, P, P, S, P, P, P, P, P]
    L.hybrid_paged_attn_workspace_bytes.argtypes = [cfgp, pgp, I]
    L.hybrid_paged_attn_workspace_bytes.restype = S
    L.hybrid_paged_attn.argtypes = [cfgp, pgp, P, P, P, P, P, I, I, I, P, P, S, P]
    L.hybrid_qk_norm_rope_cache_quant.argtypes = [cfgp, ropep, pgp, P, S, P, S, P, S, I, P, P, P, P, P, P, P, P, P, P, P]
    L.hybrid_cache_dequant.argtypes = [cfgp, pgp, P, P, P, P, P, I, P, P, P]
    L.hybrid_paged_attn_quant_workspace_bytes.argtypes = [cfgp, pgp, I]
    L.hybrid_paged_attn_quant_workspace_bytes.restype = S
    L.hybrid_paged_attn_quant.argtypes = [cfgp, pgp, P, P, P, P, P, P, P, I, I, I, P, P, S, P]
    for name in EXPORTED:
        if name not in ("hybrid_state_bytes", "hybrid_status_str", "hybrid_train_workspace_bytes",
                        "hybrid_qk_norm_rope_workspace_bytes", "hybrid_paged_attn_workspace_bytes",
                        "hybrid_paged_attn_quant_workspace_bytes"):
            getattr(L, name).restype = ctypes.c_int
    if path == _build.LIB_PATH:
        _lib = L
    return L


def make_cfg(head_dim, feat_dim, n_q_heads, n_kv_heads, block_size, io_dtype) -> hybrid_cfg:
    if not isinstance(io_dtype, int):
        import torch
        io_dtype = HYBRID_BF16 if io_dtype == torch.bfloat16 else HYBRID_F32
    return hybrid_cfg(head_dim, feat_dim, n_q_heads, n_kv_heads, block_size, io_dtype)


def _ptr(x):
    if x is None or isinstance(x, int):
        return x
    return x.data_ptr()


_raw_stream = None


def _stream(stream):
    """The raw stream to launch on; None is torch's current stream of the current device."""
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            import torch
            torch.cuda.current_stream()      # initialises CUDA, or raises without a device
            get, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
            # (building torch's stream object would take longer than the launch)
            _raw_stream = lambda: get(device())  # noqa: E731
        return _raw_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ret(status, what, check):
    if check and status != HYBRID_OK:
        raise HybridError(status, what)
    return status


def hybrid_status_str(status: int) -> str:
    return lib().hybrid_status_str(int(status)).decode()


def hybrid_state_bytes(cfg: hybrid_cfg) -> int:
    return int(lib().hybrid_state_bytes(ctypes.byref(cfg)))


def hybrid_state_init(cfg, state_ptrs, n_req, stream=None, check=True):
    st = lib().hybrid_state_init(ctypes.byref(cfg), _ptr(state_ptrs), int(n_req), _stream(stream))
    return _ret(st, "hybrid_state_init", check)


def hybrid_feature_map(cfg, X, n_rows, n_heads_x, W, Phi, stream=None, check=True):
    st = lib().hybrid_feature_map(ctypes.byref(cfg), _ptr(X), int(n_rows), int(n_heads_x), _ptr(W),
                                  _ptr(Phi), _stream(stream))
    return _ret(st, "hybrid_feature_map", check)


def hybrid_block_attn(cfg, Q, K, V, W, alpha, state_ptrs, n_req, O, stream=None, check=True):
    st = lib().hybrid_block_attn(ctypes.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(W), _ptr(alpha),
                                 _ptr(state_ptrs), int(n_req), _ptr(O), _stream(stream))
    return _ret(st, "hybrid_block_attn", check)


def hybrid_block_attn_commit(cfg, Q, K, V, W, alpha, state_ptrs, n_req, O, stream=None, check=True):
    st = lib().hybrid_block_attn_commit(ctypes.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(W),
                                        _ptr(alpha), _ptr(state_ptrs), int(n_req), _ptr(O),
                                        _stream(stream))
    return _ret(st, "hybrid_block_attn_commit", check)


def hybrid_block_attn_commit_logical(cfg, Q, K, V, W, alpha, S_logical, z_logical, n_req, O, stream=None,
                                     check=True):
    st = lib().hybrid_block_attn_commit_logical(ctypes.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(W),
                                                _ptr(alpha), _ptr(S_logical), _ptr(z_logical), int(n_req),
                                                _ptr(O), _stream(stream))
    return _ret(st, "hybrid_block_attn_commit_logical", check)


def hybrid_commit_block(cfg, K, V, n_tok, W, state_ptrs, n_req, stream=None, check=True):
    st = lib().hybrid_commit_block(ctypes.byref(cfg), _ptr(K), _ptr(V), int(n_tok), _ptr(W),
                                   _ptr(state_ptrs), int(n_req), _stream(stream))
    return _ret(st, "hybrid_commit_block", check)


def hybrid_commit_ragged(cfg, K, V, tok_offsets, W, state_ptrs, n_req, stream=None, check=True):
    """Prompt prefill with per-request lengths: request r folds rows
    tok_offsets[r]:tok_offsets[r + 1] of the packed K, V [total, Hkv, d]."""
    offs = [int(x) for x in tok_offsets]
    if len(offs) != int(n_req) + 1:
        raise ValueError(f"tok_offsets needs n_req + 1 = {int(n_req) + 1} entries, got {len(offs)}")
    arr = (ctypes.c_int * len(offs))(*offs)
    st = lib().hybrid_commit_ragged(ctypes.byref(cfg), _ptr(K), _ptr(V), arr, int(n_req), _ptr(W),
                                    _ptr(state_ptrs), _stream(stream))
    return _ret(st, "hybrid_commit_ragged", check)


def hybrid_state_unpack(cfg, state_ptrs, n_req, S_logical, z_logical, stream=None, check=True):
    st = lib().hybrid_state_unpack(ctypes.byref(cfg), _ptr(state_ptrs), int(n_req), _ptr(S_logical),
                                   _ptr(z_logical), _stream(stream))
    return _ret(st, "hybrid_state_unpack", check)


def hybrid_state_pack(cfg, S_logical, z_logical, state_ptrs, n_req, stream=None, check=True):
    st = lib().hybrid_state_pack(ctypes.byref(cfg), _ptr(S_logical), _ptr(z_logical), _ptr(state_ptrs),
                                 int(n_req), _stream(stream))
    return _ret(st, "hybrid_state_pack", check)


def hybrid_train_workspace_bytes(cfg, n_seq, seq_len) -> int:
    return int(lib().hybrid_train_workspace_bytes(ctypes.byref(cfg), int(n_seq), int(seq_len)))


def hybrid_train_forward(cfg, Q, K, V, W, alpha, n_seq, seq_len, O, workspace, workspace_bytes, stream=None,
                         check=True):
    st = lib().hybrid_train_forward(ctypes.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(W), _ptr(alpha),
                                    int(n_seq), int(seq_len), _ptr(O), _ptr(workspace), int(workspace_bytes),
                                    _stream(stream))
    return _ret(st, "hybrid_train_forward", check)


def hybrid_train_backward(cfg, Q, K, V, W, alpha, dO, n_seq, seq_len, workspace, workspace_bytes, dW, dalpha,
                          stream=None, check=True):
    st = lib().hybrid_train_backward(ctypes.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(W), _ptr(alpha),
                                     _ptr(dO), int(n_seq), int(seq_len), _ptr(workspace),
                                     int(workspace_bytes), _ptr(dW), _ptr(dalpha), _stream(stream))
    return _ret(st, "hybrid_train_backward", check)


def hybrid_debug_arm_wait_timeout(wait_ns, check=True):
    """Test hook: the next persistent step launch gives up its waits after
    wait_ns nanoseconds and withholds one barrier arrival (see hybrid.h)."""
    st = lib().hybrid_debug_arm_wait_timeout(int(wait_ns))
    return _ret(st, "hybrid_debug_arm_wait_timeout", check)


def hybrid_check(stream=None, check=True):
    st = lib().hybrid_check(_stream(stream))
    return _ret(st, "hybrid_check", check)


# ---------------------------------------------------------------- softmax layers

def make_page_cfg(page_size, n_pages, max_pages) -> hybrid_page_cfg:
    return hybrid_page_cfg(int(page_size), int(n_pages), int(max_pages))


def make_rope(rot_dim, interleaved=False, eps=1e-6, base=10000.0, kind=HYBRID_ROPE_NONE, factor=1.0, orig_len=4096.0,
              beta_fast=32.0, beta_slow=1.0, device="cuda"):
    """The rotation of a model's layers: (hybrid_rope_cfg, freqs), freqs an int64
    tensor that holds hybrid_rope_freqs' 64-bit fractions.  Made once per model.  (YaRN's ramp
    is linear in a pair's turns over orig_len; for one linear in the pair's index, bring freqs.)"""
    import torch
    arr = (ctypes.c_ulonglong * max(1, int(rot_dim) // 2))()
    scale = ctypes.c_float(1.0)
    if rot_dim:
        sc = hybrid_rope_scaling(int(kind), float(base), float(factor), float(orig_len), float(beta_fast), float(beta_slow))
        hybrid_rope_freqs(sc, rot_dim, arr, scale)
    freqs = torch.frombuffer(bytearray(arr), dtype=torch.int64).to(device)
    return hybrid_rope_cfg(int(rot_dim), int(bool(interleaved)), scale.value, float(eps)), freqs


def hybrid_page_append(pg, n_req, lens, n_new, free_pages, ring_in, block_table, slots, positions, n_slots, tok_offsets,
                       lens_out, ring_out, stream=None, check=True):
    st = lib().hybrid_page_append(pg, n_req, _ptr(lens), _ptr(n_new), _ptr(free_pages), _ptr(ring_in),
                                  _ptr(block_table), _ptr(slots), _ptr(positions), n_slots, _ptr(tok_offsets),
                                  _ptr(lens_out), _ptr(ring_out), _stream(stream))
    return _ret(st, "hybrid_page_append", check)


def hybrid_page_release(pg, n_req, rows, n_rows, lens, block_table, free_pages, ring_in, ring_out, stream=None,
                        check=True):
    st = lib().hybrid_page_release(pg, n_req, _ptr(rows), n_rows, _ptr(lens), _ptr(block_table), _ptr(free_pages),
                                   _ptr(ring_in), _ptr(ring_out), _stream(stream))
    return _ret(st, "hybrid_page_release", check)


def hybrid_rope_freqs(scaling, rot_dim, freqs, scale, check=True):
    """freqs: a ctypes array of rot_dim / 2 unsigned long long, scale: a ctypes float; both written."""
    st = lib().hybrid_rope_freqs(ctypes.byref(scaling), int(rot_dim), freqs, ctypes.byref(scale))
    return _ret(st, "hybrid_rope_freqs", check)


def hybrid_qk_norm_rope(cfg, rope, Q, q_stride, K, k_stride, n_tok, wq, wk, positions, freqs, Qo, Ko, stream=None,
                        check=True):
    st = lib().hybrid_qk_norm_rope(cfg, rope, _ptr(Q), q_stride, _ptr(K), k_stride, n_tok, _ptr(wq), _ptr(wk),
                                   _ptr(positions), _ptr(freqs), _ptr(Qo), _ptr(Ko), _stream(stream))
    return _ret(st, "hybrid_qk_norm_rope", check)


def hybrid_qk_norm_rope_cache(cfg, rope, pg, Q, q_stride, K, k_stride, V, v_stride, n_tok, wq, wk, positions, freqs,
                              slots, Qo, K_cache, V_cache, stream=None, check=True):
    st = lib().hybrid_qk_norm_rope_cache(cfg, rope, pg, _ptr(Q), q_stride, _ptr(K), k_stride, _ptr(V), v_stride, n_tok,
                                         _ptr(wq), _ptr(wk), _ptr(positions), _ptr(freqs), _ptr(slots), _ptr(Qo),
                                         _ptr(K_cache), _ptr(V_cache), _stream(stream))
    return _ret(st, "hybrid_qk_norm_rope_cache", check)


def hybrid_qk_norm_rope_workspace_bytes(cfg, n_tok) -> int:
    return int(lib().hybrid_qk_norm_rope_workspace_bytes(cfg, n_tok))


def hybrid_qk_norm_rope_backward(cfg, rope, Q, q_stride, K, k_stride, dQo, dKo, n_tok, wq, wk, positions, freqs,
                                 workspace, workspace_bytes, dQ, dK, dwq, dwk, stream=None, check=True):
    st = lib().hybrid_qk_norm_rope_backward(cfg, rope, _ptr(Q), q_stride, _ptr(K), k_stride, _ptr(dQo), _ptr(dKo),
                                            n_tok, _ptr(wq), _ptr(wk), _ptr(positions), _ptr(freqs), _ptr(workspace),
                                            workspace_bytes, _ptr(dQ), _ptr(dK), _ptr(dwq), _ptr(dwk),
                                            _stream(stream))
    return _ret(st, "hybrid_qk_norm_rope_backward", check)


def hybrid_paged_attn_workspace_bytes(cfg, pg, n_req) -> int:
    return int(lib().hybrid_paged_attn_workspace_bytes(cfg, pg, n_req))


def hybrid_paged_attn(cfg, pg, Q, K_cache, V_cache, block_table, kv_len, n_req, window, n_sink, O, workspace,
                      workspace_bytes, stream=None, check=True):
    st = lib().hybrid_paged_attn(cfg, pg, _ptr(Q), _ptr(K_cache), _ptr(V_cache), _ptr(block_table), _ptr(kv_len),
                                 n_req, window, n_sink, _ptr(O), _ptr(workspace), workspace_bytes, _stream(stream))
    return _ret(st, "hybrid_paged_attn", check)


# ---------------------------------------------------------------- the cache in 8 bits

def hybrid_qk_norm_rope_cache_quant(cfg, rope, pg, Q, q_stride, K, k_stride, V, v_stride, n_tok, wq, wk, positions, freqs,
                                    slots, Qo, K_cache, V_cache, K_scale, V_scale, stream=None, check=True):
    st = lib().hybrid_qk_norm_rope_cache_quant(cfg, rope, pg, _ptr(Q), q_stride, _ptr(K), k_stride, _ptr(V), v_stride, n_tok,
                                               _ptr(wq), _ptr(wk), _ptr(positions), _ptr(freqs), _ptr(slots), _ptr(Qo),
                                               _ptr(K_cache), _ptr(V_cache), _ptr(K_scale), _ptr(V_scale), _stream(stream))
    return _ret(st, "hybrid_qk_norm_rope_cache_quant", check)


def hybrid_cache_dequant(cfg, pg, K_cache, V_cache, K_scale, V_scale, slots, n_tok, K, V, stream=None, check=True):
    st = lib().hybrid_cache_dequant(cfg, pg, _ptr(K_cache), _ptr(V_cache), _ptr(K_scale), _ptr(V_scale), _ptr(slots), n_tok,
                                    _ptr(K), _ptr(V), _stream(stream))
    return _ret(st, "hybrid_cache_dequant", check)


def hybrid_paged_attn_quant_workspace_bytes(cfg, pg, n_req) -> int:
    return int(lib().hybrid_paged_attn_quant_workspace_bytes(cfg, pg, n_req))


def hybrid_paged_attn_quant(cfg, pg, Q, K_cache, V_cache, K_scale, V_scale, block_table, kv_len, n_req, window, n_sink, O,
                            workspace, workspace_bytes, stream=None, check=True):
    st = lib().hybrid_paged_attn_quant(cfg, pg, _ptr(Q), _ptr(K_cache), _ptr(V_cache), _ptr(K_scale), _ptr(V_scale),
                                       _ptr(block_table), _ptr(kv_len), n_req, window, n_sink, _ptr(O), _ptr(workspace),
                                       workspace_bytes, _stream(stream))
    return _ret(st, "hybrid_paged_attn_quant", check)
