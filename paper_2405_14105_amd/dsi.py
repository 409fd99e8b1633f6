"""ctypes binding of libdsi.so -- argument marshalling only.

Every function has the name of the C entry point it calls (include/dsi.h)
and raises DsiError on a non-zero status.  Device buffers are passed as
integer addresses or torch tensors (their data_ptr()); torch is used only
for device memory and streams.  Every step of the verification runs in the
library's HIP kernels; there is no fallback: if libdsi.so is missing or was
built for another GPU, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdsi.so")

DSI_OK, DSI_EINVAL, DSI_ENOMEM, DSI_EHIP, DSI_ECAPACITY, DSI_ESTATE = range(6)
DSI_F32, DSI_BF16 = 0, 1
DSI_SAMPLE, DSI_GREEDY = 0, 1
DSI_MAX_ROWS = 64
DSI_MAX_ATTEND_ROWS = 1024
DSI_MAX_TOP = 64
TENSOR_IDS = {
    "embed": 0, "final_norm": 1, "lm_head": 2, "attn_norm": 3, "wq": 4, "wk": 5, "wv": 6,
    "wo": 7, "ffn_norm": 8, "w_gate": 9, "w_up": 10, "w_down": 11,
}
EXPORTED = (
    "dsi_model_create", "dsi_model_set_tensor", "dsi_model_destroy", "dsi_kv_create",
    "dsi_kv_destroy", "dsi_prefill", "dsi_verify", "dsi_verify_tree", "dsi_draft", "dsi_accept",
    "dsi_accept_noalloc", "dsi_kv_bytes", "dsi_kv_wrap", "dsi_kv_fork", "dsi_attend", "dsi_logprobs_workspace",
    "dsi_logprobs", "dsi_rope_table", "dsi_rotate", "dsi_page_append", "dsi_page_attend_workspace", "dsi_page_attend",
    "dsi_adjust", "dsi_kv_rollback", "dsi_kv_poison", "dsi_kv_length", "dsi_sync", "dsi_kv_export", "dsi_kv_import", "dsi_kv_set_length",
    "dsi_profile_begin", "dsi_profile_end", "dsi_profile_kernel", "dsi_profile_stream", "dsi_last_error",
)
DSI_K_QKV, DSI_K_ATTN, DSI_K_OPROJ, DSI_K_GATEUP, DSI_K_DOWN, DSI_K_HEAD, DSI_K_VERIFY = range(1, 8)


class DsiError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"dsi status {status}: {msg}")
        self.status = status


class dsi_config(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("d_ff", ctypes.c_int32),
        ("vocab", ctypes.c_int32), ("rope_base", ctypes.c_float), ("rms_eps", ctypes.c_float),
        ("wdtype", ctypes.c_int32), ("kvdtype", ctypes.c_int32),
    ]


class dsi_verify_args(ctypes.Structure):
    _fields_ = [
        ("window0", ctypes.c_int32), ("n_windows", ctypes.c_int32), ("k", ctypes.c_int32),
        ("d_tokens", ctypes.c_void_p), ("d_q", ctypes.c_void_p), ("d_u", ctypes.c_void_p),
        ("temperature", ctypes.c_float), ("mode", ctypes.c_int32), ("commit", ctypes.c_int32),
        ("d_logits_out", ctypes.c_void_p), ("d_hidden_out", ctypes.c_void_p),
    ]


class dsi_tree_args(ctypes.Structure):
    _fields_ = [
        ("window0", ctypes.c_int32), ("n_windows", ctypes.c_int32), ("n_nodes", ctypes.c_int32),
        ("d_tokens", ctypes.c_void_p), ("d_parent", ctypes.c_void_p), ("commit", ctypes.c_int32),
        ("d_logits_out", ctypes.c_void_p),
    ]


class dsi_attend_args(ctypes.Structure):
    _fields_ = [
        ("layer", ctypes.c_int32), ("window0", ctypes.c_int32), ("n_windows", ctypes.c_int32),
        ("rows", ctypes.c_int32), ("d_q", ctypes.c_void_p), ("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p),
        ("commit", ctypes.c_int32), ("d_out", ctypes.c_void_p),
    ]


class dsi_logprobs_args(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("n_top", ctypes.c_int32),
        ("ld", ctypes.c_int64), ("d_logits", ctypes.c_void_p), ("d_targets", ctypes.c_void_p),
        ("temperature", ctypes.c_float), ("d_logprob", ctypes.c_void_p), ("d_entropy", ctypes.c_void_p),
        ("d_top_ids", ctypes.c_void_p), ("d_top_logprobs", ctypes.c_void_p), ("d_ws", ctypes.c_void_p),
        ("ws_bytes", ctypes.c_size_t),
    ]


DSI_ROPE_HALF, DSI_ROPE_PAIRS = 0, 1
DSI_ROPE_PLAIN, DSI_ROPE_LINEAR, DSI_ROPE_BASE, DSI_ROPE_BANDS, DSI_ROPE_RAMP = range(5)


class dsi_rope_spec(ctypes.Structure):
    _fields_ = [
        ("dim", ctypes.c_int32), ("scaling", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
        ("low", ctypes.c_double), ("high", ctypes.c_double), ("context", ctypes.c_double),
    ]


class dsi_rope(ctypes.Structure):
    _fields_ = [
        ("style", ctypes.c_int32), ("dim", ctypes.c_int32), ("d_freq", ctypes.c_void_p), ("gain", ctypes.c_float),
    ]


class dsi_rotate_args(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("ld_q", ctypes.c_int64), ("ld_k", ctypes.c_int64),
        ("ld_q_out", ctypes.c_int64), ("ld_k_out", ctypes.c_int64), ("d_q", ctypes.c_void_p), ("d_k", ctypes.c_void_p),
        ("d_pos", ctypes.c_void_p), ("d_gain_q", ctypes.c_void_p), ("d_gain_k", ctypes.c_void_p),
        ("eps", ctypes.c_float), ("rope", dsi_rope), ("d_q_out", ctypes.c_void_p), ("d_k_out", ctypes.c_void_p),
    ]


class dsi_pages(ctypes.Structure):
    _fields_ = [
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("kvdtype", ctypes.c_int32),
        ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p),
        ("n_windows", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("d_table", ctypes.c_void_p),
        ("d_len", ctypes.c_void_p), ("d_row0", ctypes.c_void_p),
    ]


class dsi_page_append_args(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("dtype", ctypes.c_int32), ("ld_q", ctypes.c_int64),
        ("ld_k", ctypes.c_int64), ("ld_v", ctypes.c_int64), ("ld_q_out", ctypes.c_int64), ("d_q", ctypes.c_void_p),
        ("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p), ("d_pos", ctypes.c_void_p), ("d_gain_q", ctypes.c_void_p),
        ("d_gain_k", ctypes.c_void_p), ("eps", ctypes.c_float), ("rope", dsi_rope), ("d_q_out", ctypes.c_void_p),
    ]


class dsi_page_attend_args(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reach", ctypes.c_int32),
        ("ld_q", ctypes.c_int64), ("ld_out", ctypes.c_int64), ("d_q", ctypes.c_void_p), ("scale", ctypes.c_float),
        ("d_out", ctypes.c_void_p), ("d_ws", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t),
    ]


class dsi_adjust_args(ctypes.Structure):
    _fields_ = [
        ("n_windows", ctypes.c_int32), ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("n_bias", ctypes.c_int32), ("ld", ctypes.c_int64), ("ld_out", ctypes.c_int64), ("ld_seen", ctypes.c_int64),
        ("ld_allowed", ctypes.c_int64), ("d_logits", ctypes.c_void_p), ("d_seen", ctypes.c_void_p),
        ("d_n_seen", ctypes.c_void_p), ("d_tokens", ctypes.c_void_p), ("d_repetition", ctypes.c_void_p),
        ("d_frequency", ctypes.c_void_p), ("d_presence", ctypes.c_void_p), ("d_bias_ids", ctypes.c_void_p),
        ("d_bias", ctypes.c_void_p), ("d_allowed", ctypes.c_void_p), ("d_out", ctypes.c_void_p),
    ]


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libdsi.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2405_14105_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32, SZ, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
    PP = ctypes.POINTER(ctypes.c_void_p)
    sig = {
        "dsi_model_create": ([ctypes.POINTER(dsi_config), P, PP], I32),
        "dsi_model_set_tensor": ([P, I32, I32, P, SZ, I32], I32),
        "dsi_model_destroy": ([P], I32),
        "dsi_kv_create": ([P, I32, I32, PP], I32),
        "dsi_kv_destroy": ([P], I32),
        "dsi_prefill": ([P, P, I32, P, I32, P], I32),
        "dsi_verify": ([P, P, ctypes.POINTER(dsi_verify_args), P, P], I32),
        "dsi_verify_tree": ([P, P, ctypes.POINTER(dsi_tree_args), P, P, P], I32),
        "dsi_draft": ([P, P, I32, P, I32, I32, P, F, P, P], I32),
        "dsi_accept": ([P, I32, I32, I32, P, P, P, P, F, I32, P, P], I32),
        "dsi_accept_noalloc": ([P, I32, I32, I32, P, P, P, P, F, I32, P, P], I32),
        "dsi_kv_bytes": ([P, I32, I32, ctypes.POINTER(SZ)], I32),
        "dsi_kv_wrap": ([P, I32, I32, P, P, SZ, PP], I32),
        "dsi_kv_fork": ([P, I32, I32, I32, I32], I32),
        "dsi_attend": ([P, P, ctypes.POINTER(dsi_attend_args)], I32),
        "dsi_logprobs_workspace": ([I32, I32, I32, ctypes.POINTER(SZ)], I32),
        "dsi_logprobs": ([P, ctypes.POINTER(dsi_logprobs_args)], I32),
        "dsi_rope_table": ([ctypes.POINTER(dsi_rope_spec), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(F)], I32),
        "dsi_rotate": ([P, ctypes.POINTER(dsi_rotate_args)], I32),
        "dsi_page_append": ([P, ctypes.POINTER(dsi_pages), ctypes.POINTER(dsi_page_append_args)], I32),
        "dsi_page_attend_workspace": ([ctypes.POINTER(dsi_pages), I32, I32, ctypes.POINTER(SZ)], I32),
        "dsi_page_attend": ([P, ctypes.POINTER(dsi_pages), ctypes.POINTER(dsi_page_attend_args)], I32),
        "dsi_adjust": ([P, ctypes.POINTER(dsi_adjust_args)], I32),
        "dsi_kv_rollback": ([P, I32, I32], I32),
        "dsi_kv_poison": ([P, I32], I32),
        "dsi_kv_length": ([P, I32, ctypes.POINTER(ctypes.c_int32)], I32),
        "dsi_sync": ([P], I32),
        "dsi_kv_export": ([P, I32, I32, I32, P, P], I32),
        "dsi_kv_import": ([P, I32, I32, I32, P, P], I32),
        "dsi_kv_set_length": ([P, I32, I32], I32),
        "dsi_profile_begin": ([P, I32], I32),
        "dsi_profile_end": ([P, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_double)], I32),
        "dsi_profile_kernel": ([P, P, I32, I32, ctypes.POINTER(ctypes.c_int32),
                                ctypes.POINTER(ctypes.c_double)], I32),
        "dsi_profile_stream": ([P, ctypes.c_uint64, I32, I32, I32, I32, P, ctypes.POINTER(ctypes.c_uint64),
                                ctypes.POINTER(ctypes.c_double)], I32),
        "dsi_last_error": ([], ctypes.c_char_p),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def _ptr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _check(st: int):
    if st != DSI_OK:
        raise DsiError(st, load().dsi_last_error().decode())


def make_config(n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff, vocab, rope_base=10000.0,
                rms_eps=1e-5, wdtype=DSI_BF16, kvdtype=DSI_BF16) -> dsi_config:
    return dsi_config(n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff, vocab, rope_base,
                      rms_eps, wdtype, kvdtype)


def dsi_model_create(cfg: dsi_config, stream: int = 0) -> int:
    out = ctypes.c_void_p()
    _check(load().dsi_model_create(ctypes.byref(cfg), stream or None, ctypes.byref(out)))
    return out.value


def dsi_model_set_tensor(model: int, layer: int, tensor_id: int, src, nbytes: int, src_on_device: bool):
    _check(load().dsi_model_set_tensor(model, layer, tensor_id, src, nbytes, int(src_on_device)))


def dsi_model_destroy(model: int):
    _check(load().dsi_model_destroy(model))


def dsi_kv_create(model: int, n_windows: int, max_len: int) -> int:
    out = ctypes.c_void_p()
    _check(load().dsi_kv_create(model, n_windows, max_len, ctypes.byref(out)))
    return out.value


def dsi_kv_destroy(kv: int):
    _check(load().dsi_kv_destroy(kv))


def dsi_prefill(model: int, kv: int, window: int, d_tokens, n: int, d_last_logits=None):
    _check(load().dsi_prefill(model, kv, window, _ptr(d_tokens), n, _ptr(d_last_logits)))


def dsi_verify(model: int, kv: int, window0: int, n_windows: int, k: int, d_tokens, d_q, d_u,
               d_n_accepted, d_next_token, temperature: float = 1.0, mode: int = DSI_SAMPLE,
               commit: bool = True, d_logits_out=None, d_hidden_out=None):
    a = dsi_verify_args(window0, n_windows, k, _ptr(d_tokens), _ptr(d_q), _ptr(d_u), temperature,
                        mode, int(commit), _ptr(d_logits_out), _ptr(d_hidden_out))
    _check(load().dsi_verify(model, kv, ctypes.byref(a), _ptr(d_n_accepted), _ptr(d_next_token)))


def dsi_verify_tree(model: int, kv: int, window0: int, n_windows: int, n_nodes: int, d_tokens, d_parent,
                    d_path, d_n_accepted, d_next_token, commit: bool = True, d_logits_out=None):
    a = dsi_tree_args(window0, n_windows, n_nodes, _ptr(d_tokens), _ptr(d_parent), int(commit),
                      _ptr(d_logits_out))
    _check(load().dsi_verify_tree(model, kv, ctypes.byref(a), _ptr(d_path), _ptr(d_n_accepted),
                                  _ptr(d_next_token)))


def dsi_draft(model: int, kv: int, window: int, d_feed, n_feed: int, k: int, d_u, d_tokens, d_q,
              temperature: float = 1.0):
    _check(load().dsi_draft(model, kv, window, _ptr(d_feed), n_feed, k, _ptr(d_u), temperature,
                            _ptr(d_tokens), _ptr(d_q)))


def dsi_accept(stream: int, n_windows: int, k: int, vocab: int, d_logits, d_tokens, d_q, d_u,
               d_n_accepted, d_next_token, temperature: float = 1.0, mode: int = DSI_SAMPLE):
    _check(load().dsi_accept(stream or None, n_windows, k, vocab, _ptr(d_logits), _ptr(d_tokens),
                             _ptr(d_q), _ptr(d_u), temperature, mode, _ptr(d_n_accepted),
                             _ptr(d_next_token)))


def dsi_accept_noalloc(stream: int, n_windows: int, k: int, vocab: int, d_logits, d_tokens, d_q, d_u,
                       d_n_accepted, d_next_token, temperature: float = 1.0, mode: int = DSI_SAMPLE):
    _check(load().dsi_accept_noalloc(stream or None, n_windows, k, vocab, _ptr(d_logits), _ptr(d_tokens),
                                     _ptr(d_q), _ptr(d_u), temperature, mode, _ptr(d_n_accepted),
                                     _ptr(d_next_token)))


def dsi_kv_bytes(model: int, n_windows: int, max_len: int) -> int:
    """Bytes of such a cache's keys (and of its values)."""
    out = ctypes.c_size_t()
    _check(load().dsi_kv_bytes(model, n_windows, max_len, ctypes.byref(out)))
    return out.value


def dsi_kv_wrap(model: int, n_windows: int, max_len: int, d_k, d_v, nbytes: int) -> int:
    out = ctypes.c_void_p()
    _check(load().dsi_kv_wrap(model, n_windows, max_len, _ptr(d_k), _ptr(d_v), nbytes, ctypes.byref(out)))
    return out.value


def dsi_kv_fork(kv: int, src: int, window0: int, n_windows: int, length: int = -1):
    _check(load().dsi_kv_fork(kv, src, window0, n_windows, length))


def dsi_attend(model: int, kv: int, layer: int, window0: int, n_windows: int, rows: int, d_q, d_k, d_v, d_out,
               commit: bool = False):
    a = dsi_attend_args(layer, window0, n_windows, rows, _ptr(d_q), _ptr(d_k), _ptr(d_v), int(commit), _ptr(d_out))
    _check(load().dsi_attend(model, kv, ctypes.byref(a)))


def dsi_logprobs_workspace(rows: int, vocab: int, n_top: int) -> int:
    """Bytes of the workspace that dsi_logprobs needs for these sizes."""
    out = ctypes.c_size_t()
    _check(load().dsi_logprobs_workspace(rows, vocab, n_top, ctypes.byref(out)))
    return out.value


def dsi_logprobs(stream: int, rows: int, vocab: int, d_logits, d_targets, n_top: int, d_logprob, d_entropy, d_top_ids,
                 d_top_logprobs, d_ws, ws_bytes: int, temperature: float = 1.0, dtype: int = DSI_F32, ld: int = 0):
    """ld: entries from one row of logits to the next (0: vocab)."""
    a = dsi_logprobs_args(rows, vocab, dtype, n_top, ld or vocab, _ptr(d_logits), _ptr(d_targets), temperature,
                          _ptr(d_logprob), _ptr(d_entropy), _ptr(d_top_ids), _ptr(d_top_logprobs), _ptr(d_ws), ws_bytes)
    _check(load().dsi_logprobs(stream or None, ctypes.byref(a)))


def make_rope(dim: int, d_freq, gain: float = 1.0, style: int = DSI_ROPE_HALF) -> dsi_rope:
    return dsi_rope(style, dim, _ptr(d_freq), gain)


def dsi_rope_table(dim: int, base: float = 10000.0, scaling: int = DSI_ROPE_PLAIN, factor: float = 1.0, low: float = 1.0,
                   high: float = 32.0, context: float = 0.0):
    """Returns (radians per position of each rotated pair, as a list; gain)."""
    freq, gain = (ctypes.c_double * max(1, dim // 2))(), ctypes.c_float()
    spec = dsi_rope_spec(dim, scaling, base, factor, low, high, context)
    _check(load().dsi_rope_table(ctypes.byref(spec), freq, ctypes.byref(gain)))
    return list(freq), gain.value


def dsi_rotate(stream: int, rows: int, n_heads: int, n_kv_heads: int, head_dim: int, d_q, d_k, d_pos, d_q_out, d_k_out,
               rope: dsi_rope, dtype: int = DSI_F32, ld_q: int = 0, ld_k: int = 0, ld_q_out: int = 0, ld_k_out: int = 0,
               d_gain_q=None, d_gain_k=None, eps: float = 1e-5):
    """ld_*: entries from one row to the next (0: its heads and nothing else)."""
    nq, nk = n_heads * head_dim, n_kv_heads * head_dim
    a = dsi_rotate_args(rows, n_heads, n_kv_heads, head_dim, dtype, ld_q or nq, ld_k or nk, ld_q_out or nq, ld_k_out or nk,
                        _ptr(d_q), _ptr(d_k), _ptr(d_pos), _ptr(d_gain_q), _ptr(d_gain_k), eps, rope, _ptr(d_q_out),
                        _ptr(d_k_out))
    _check(load().dsi_rotate(stream or None, ctypes.byref(a)))


def make_pages(n_kv_heads: int, head_dim: int, kvdtype: int, n_pages: int, page_size: int, d_k, d_v, n_windows: int,
               max_pages: int, d_table, d_len, d_row0) -> dsi_pages:
    """The tensors must live as long as calls use what is returned."""
    return dsi_pages(n_kv_heads, head_dim, kvdtype, n_pages, page_size, _ptr(d_k), _ptr(d_v), n_windows, max_pages,
                     _ptr(d_table), _ptr(d_len), _ptr(d_row0))


def dsi_page_append(stream: int, pages: dsi_pages, rows: int, n_heads: int, d_q, d_k, d_v, d_q_out, rope: dsi_rope,
                    dtype: int = DSI_F32, ld_q: int = 0, ld_k: int = 0, ld_v: int = 0, ld_q_out: int = 0, d_pos=None,
                    d_gain_q=None, d_gain_k=None, eps: float = 1e-5):
    nq, nk = n_heads * pages.head_dim, pages.n_kv_heads * pages.head_dim
    a = dsi_page_append_args(rows, n_heads, dtype, ld_q or nq, ld_k or nk, ld_v or nk, ld_q_out or nq, _ptr(d_q), _ptr(d_k),
                             _ptr(d_v), _ptr(d_pos), _ptr(d_gain_q), _ptr(d_gain_k), eps, rope, _ptr(d_q_out))
    _check(load().dsi_page_append(stream or None, ctypes.byref(pages), ctypes.byref(a)))


def dsi_page_attend_workspace(pages: dsi_pages, rows: int, n_heads: int) -> int:
    """Bytes of the workspace that dsi_page_attend needs for these sizes."""
    out = ctypes.c_size_t()
    _check(load().dsi_page_attend_workspace(ctypes.byref(pages), rows, n_heads, ctypes.byref(out)))
    return out.value


def dsi_page_attend(stream: int, pages: dsi_pages, rows: int, n_heads: int, d_q, d_out, d_ws, ws_bytes: int,
                    dtype: int = DSI_F32, reach: int = 0, ld_q: int = 0, ld_out: int = 0, scale: float = 0.0):
    n = n_heads * pages.head_dim
    a = dsi_page_attend_args(rows, n_heads, dtype, reach, ld_q or n, ld_out or n, _ptr(d_q), scale, _ptr(d_out), _ptr(d_ws),
                             ws_bytes)
    _check(load().dsi_page_attend(stream or None, ctypes.byref(pages), ctypes.byref(a)))


def dsi_adjust(stream: int, n_windows: int, rows: int, vocab: int, d_logits, d_out, dtype: int = DSI_F32, ld: int = 0,
               ld_out: int = 0, d_seen=None, d_n_seen=None, ld_seen: int = 0, d_tokens=None, d_repetition=None,
               d_frequency=None, d_presence=None, n_bias: int = 0, d_bias_ids=None, d_bias=None, d_allowed=None,
               ld_allowed: int = 0):
    """ld, ld_out: 0: vocab; ld_allowed: 0: (vocab + 31) // 32 words."""
    a = dsi_adjust_args(n_windows, rows, vocab, dtype, n_bias, ld or vocab, ld_out or vocab, ld_seen,
                        ld_allowed or (vocab + 31) // 32, _ptr(d_logits), _ptr(d_seen), _ptr(d_n_seen), _ptr(d_tokens),
                        _ptr(d_repetition), _ptr(d_frequency), _ptr(d_presence), _ptr(d_bias_ids) if n_bias else None,
                        _ptr(d_bias) if n_bias else None, _ptr(d_allowed), _ptr(d_out))
    _check(load().dsi_adjust(stream or None, ctypes.byref(a)))


def dsi_kv_rollback(kv: int, window: int, new_len: int):
    _check(load().dsi_kv_rollback(kv, window, new_len))


def dsi_kv_poison(kv: int, window: int):
    _check(load().dsi_kv_poison(kv, window))


def dsi_kv_length(kv: int, window: int) -> int:
    out = ctypes.c_int32()
    _check(load().dsi_kv_length(kv, window, ctypes.byref(out)))
    return out.value


def dsi_sync(model: int):
    _check(load().dsi_sync(model))


def dsi_kv_export(kv: int, window: int, layer: int, length: int, d_k, d_v):
    _check(load().dsi_kv_export(kv, window, layer, length, _ptr(d_k), _ptr(d_v)))


def dsi_kv_import(kv: int, window: int, layer: int, length: int, d_k, d_v):
    _check(load().dsi_kv_import(kv, window, layer, length, _ptr(d_k), _ptr(d_v)))


def dsi_kv_set_length(kv: int, window: int, length: int):
    _check(load().dsi_kv_set_length(kv, window, length))


def dsi_profile_begin(model: int, kernel_class: int):
    _check(load().dsi_profile_begin(model, kernel_class))


def dsi_profile_end(model: int):
    """Returns (launches, total_ms)."""
    n = ctypes.c_int32()
    t = ctypes.c_double()
    _check(load().dsi_profile_end(model, ctypes.byref(n), ctypes.byref(t)))
    return n.value, t.value


def dsi_profile_kernel(model: int, kv: int, kernel_class: int, rounds: int = 3):
    """Returns (launches, avg_ms) of one GEMM class replayed back to back."""
    n = ctypes.c_int32()
    t = ctypes.c_double()
    _check(load().dsi_profile_kernel(model, kv, kernel_class, rounds, ctypes.byref(n), ctypes.byref(t)))
    return n.value, t.value


def dsi_profile_stream(d_buf, nbytes: int, slices: int, nontemporal: bool, rounds: int, d_sink,
                       workgroups: int = 0):
    """Returns (bytes per launch, avg_ms) of the library's streaming read over
    `slices` slices of the device buffer d_buf, one per launch in turn, with
    `workgroups` workgroups of 8 waves (0: the default 256)."""
    b = ctypes.c_uint64()
    t = ctypes.c_double()
    _check(load().dsi_profile_stream(_ptr(d_buf), nbytes, slices, int(bool(nontemporal)), workgroups, rounds,
                                     _ptr(d_sink), ctypes.byref(b), ctypes.byref(t)))
    return b.value, t.value


def dsi_last_error() -> str:
    return load().dsi_last_error().decode()
