"""Python binding of libflasheval (ctypes).  Argument marshalling only: every step of the pass
runs in the library's HIP kernels.  Functions carry the names of the C ABI in
include/flasheval.h and take torch tensors that live on the current HIP device; the stream is
torch's current stream unless one is given.

There is no fallback: if libflasheval.so has not been built, `load_library` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence, Tuple

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libflasheval.so")

FE_OK, FE_EINVAL, FE_EUNSUPPORTED, FE_ENOMEM, FE_EHIP = range(5)
FE_F32, FE_BF16 = 0, 1
FE_ATTN_SOFTMAX, FE_ATTN_LINEAR = 0, 1
FE_DEV_BAD_INDEX, FE_DEV_BAD_TOKEN, FE_DEV_BAD_PAGE = 1, 2, 4
FE_LOSS_MSE, FE_LOSS_BCE, FE_LOSS_CE = 0, 1, 2
LOSS_KIND = {"mse": FE_LOSS_MSE, "bce": FE_LOSS_BCE, "ce": FE_LOSS_CE}

EXPORTED = ("fe_param_count", "fe_model_create", "fe_model_destroy", "fe_workspace_size", "fe_kv_size", "fe_last_error",
            "fe_read_device_status", "fe_encode_context", "fe_encode_items", "fe_assemble", "fe_cross_sequence",
            "fe_cross_sequence_noalloc", "fe_score_select", "fe_encode_sequences", "fe_score_objectives", "fe_naive_workspace_size", "fe_evaluate_naive", "fe_trace_enable", "fe_trace_read",
            "fe_trace_read_launches", "fe_trace_family", "fe_train_workspace_size", "fe_train_grads",
            "fe_executor_create", "fe_executor_submit", "fe_executor_join", "fe_executor_destroy",
            "fe_cache_append", "fe_prefix_workspace_size", "fe_prefix_attention", "fe_prefix_attention_grad",
            "fe_packed_page_bytes", "fe_packed_append", "fe_packed_read", "fe_packed_attention", "fe_packed_weights",
            "fe_packed_weights_strided", "fe_packed_evict", "fe_packed_workspace_size")
FE_EXECUTOR_MAX_STREAMS = 8
FE_TRACE_FAMILIES = 12


class FeError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        super().__init__(f"{where} -> status {status}: {msg}")
        self.status = status


class fe_config(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("ffn_dim", ctypes.c_int32), ("max_L", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("attention", ctypes.c_int32)]


class fe_pass_args(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("M", ctypes.c_int32), ("K", ctypes.c_int32),
                ("L", ctypes.c_int32), ("x", ctypes.c_void_p), ("ctx_ids", ctypes.c_void_p), ("pool", ctypes.c_void_p),
                ("lists", ctypes.c_void_p), ("kv", ctypes.c_void_p), ("uniq", ctypes.c_void_p),
                ("n_uniq", ctypes.c_void_p), ("slot", ctypes.c_void_p), ("H", ctypes.c_void_p), ("seq", ctypes.c_void_p),
                ("Cp", ctypes.c_void_p), ("scores", ctypes.c_void_p), ("best", ctypes.c_void_p), ("ws", ctypes.c_void_p),
                ("ws_bytes", ctypes.c_size_t)]


def _struct(name: str, ints: str, pointers: str, tail=()):
    """A ctypes structure of int32 fields followed by pointer fields, in the order of the C header."""
    fields = [(n, ctypes.c_float if n == "scale" else ctypes.c_int32) for n in ints.split()]
    fields += [(n, ctypes.c_void_p) for n in pointers.split()]
    return type(name, (ctypes.Structure,), {"_fields_": fields + list(tail)})


fe_append_args = _struct(
    "fe_append_args",
    "dtype N S n_heads n_kv_heads dh rot neighbours page_rows n_pages table_cols q_ld k_ld v_ld q_out_ld page_ld",
    "q k v q_out freq table len new_len pos0 k_pages v_pages len_out status")
fe_prefix_args = _struct(
    "fe_prefix_args", "dtype B K S n_heads n_kv_heads dh T L page_rows n_pages causal scale q_ld ctx_ld own_ld out_ld",
    "q ctx_k ctx_v own_k own_v table ctx_len q_len own_len out lse out_rest ws", [("ws_bytes", ctypes.c_size_t)])


class fe_prefix_grads(ctypes.Structure):
    _fields_ = [("dout", ctypes.c_void_p), ("dout_ld", ctypes.c_int32), ("dq_ld", ctypes.c_int32),
                ("dctx_ld", ctypes.c_int32), ("down_ld", ctypes.c_int32), ("dq", ctypes.c_void_p),
                ("dctx_k", ctypes.c_void_p), ("dctx_v", ctypes.c_void_p), ("down_k", ctypes.c_void_p),
                ("down_v", ctypes.c_void_p)]


class fe_packed_cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("page_ld", ctypes.c_int64), ("table", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("N", ctypes.c_int32), ("cols", ctypes.c_int32), ("page_rows", ctypes.c_int32), ("n_pages", ctypes.c_int32)]


def _packed(name: str, caches: str, ints: str, pointers: str, tail=()):
    """A ctypes structure of fe_packed_cache fields, then as _struct."""
    plain = _struct(name, ints, pointers, tail)
    return type(name, (ctypes.Structure,), {"_fields_": [(n, fe_packed_cache) for n in caches.split()] + plain._fields_})


fe_packed_append_args = _packed(
    "fe_packed_append_args", "cache", "dtype S n_heads n_kv_heads dh rot neighbours q_ld k_ld v_ld q_out_ld",
    "q k v q_out freq new_len pos0 len_out status")
fe_packed_read_args = _packed("fe_packed_read_args", "cache", "dtype S n_kv_heads dh k_ld v_ld", "start count k v")
fe_packed_args = _packed(
    "fe_packed_args", "ctx own", "dtype B K S n_heads n_kv_heads dh causal scale q_ld out_ld",
    "q q_len out lse ctx_w own_w ctx_w_out own_w_out ws", [("ws_bytes", ctypes.c_size_t)])
fe_packed_evict_args = _packed(
    "fe_packed_evict_args", "from_ to", "n_kv_heads dh keep first recent", "weight weight_out kept status")

_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libflasheval.so (once).  Raises if it is missing: build it with __graft_entry__.build()."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing; build the HIP library first (python -c "
                           "'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(path)
    P, I, Z, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_int
    cfgp = ctypes.POINTER(fe_config)
    sig = {
        "fe_param_count": (S, [cfgp, ctypes.POINTER(Z)]),
        "fe_model_create": (S, [cfgp, P, Z, ctypes.POINTER(P)]),
        "fe_model_destroy": (None, [P]),
        "fe_workspace_size": (S, [P, I, I, I, I, I, ctypes.POINTER(Z)]),
        "fe_kv_size": (S, [P, I, I, ctypes.POINTER(Z)]),
        "fe_last_error": (ctypes.c_char_p, []),
        "fe_read_device_status": (S, [P, P, I, P, P]),
        "fe_encode_context": (S, [P, I, I, P, P, P, P, Z, P]),
        "fe_encode_items": (S, [P, I, I, P, P, I, I, P, I, P, P, P, P, P, Z, P]),
        "fe_assemble": (S, [P, I, I, I, I, P, P, P, P]),
        "fe_cross_sequence": (S, [P, I, I, I, P, P, P, Z, P]),
        "fe_cross_sequence_noalloc": (S, [P, I, I, I, P, P, P]),
        "fe_score_select": (S, [P, I, I, P, P, P, P]),
        "fe_encode_sequences": (S, [P, I, I, I, P, P, P, Z, P]),
        "fe_score_objectives": (S, [P, I, I, P, I, P, P, P, P, P, P, P]),
        "fe_naive_workspace_size": (S, [P, I, I, I, I, I, I, ctypes.POINTER(Z)]),
        "fe_evaluate_naive": (S, [P, I, I, I, I, I, P, P, P, P, P, P, P, P, Z, P]),
        "fe_trace_enable": (S, [I]),
        "fe_trace_read": (S, [P, P]),
        "fe_trace_read_launches": (S, [P, P, ctypes.c_int64, P]),
        "fe_trace_family": (ctypes.c_char_p, [I]),
        "fe_train_workspace_size": (S, [cfgp, I, I, I, I, I, ctypes.POINTER(Z)]),
        "fe_train_grads": (S, [cfgp, P, I, I, I, I, I, P, P, P, P, P, I, P, P, P, P, Z, P]),
        "fe_executor_create": (S, [P, I, ctypes.POINTER(P)]),
        "fe_executor_submit": (S, [P, ctypes.POINTER(fe_pass_args), P]),
        "fe_executor_join": (S, [P, P]),
        "fe_executor_destroy": (None, [P]),
        "fe_cache_append": (S, [ctypes.POINTER(fe_append_args), P]),
        "fe_prefix_workspace_size": (S, [ctypes.POINTER(fe_prefix_args), I, ctypes.POINTER(Z)]),
        "fe_prefix_attention": (S, [ctypes.POINTER(fe_prefix_args), P]),
        "fe_prefix_attention_grad": (S, [ctypes.POINTER(fe_prefix_args), ctypes.POINTER(fe_prefix_grads), P]),
        "fe_packed_page_bytes": (S, [I, I, I, ctypes.POINTER(Z)]),
        "fe_packed_append": (S, [ctypes.POINTER(fe_packed_append_args), P]),
        "fe_packed_read": (S, [ctypes.POINTER(fe_packed_read_args), P]),
        "fe_packed_workspace_size": (S, [ctypes.POINTER(fe_packed_args), I, ctypes.POINTER(Z)]),
        "fe_packed_attention": (S, [ctypes.POINTER(fe_packed_args), P]),
        "fe_packed_weights": (S, [ctypes.POINTER(fe_packed_args), P]),
        "fe_packed_weights_strided": (S, [ctypes.POINTER(fe_packed_args), ctypes.POINTER(ctypes.c_int64), P]),
        "fe_packed_evict": (S, [ctypes.POINTER(fe_packed_evict_args), P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _check(status: int, where: str) -> None:
    if status != FE_OK:
        raise FeError(status, where, load_library().fe_last_error().decode())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    import torch
    return _current_stream(torch.cuda.current_device())


def _current_stream(index: int) -> int:
    """Handle of device `index`'s current stream; without torch's own short way to it, where a build of torch has none, by a stream
    object (about a microsecond more)."""
    import torch
    short = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return short(index) if short else torch.cuda.current_stream(index).cuda_stream


# ---------------------------------------------------------------------------------------------
# Parameter order of fe_model_create (as documented in include/flasheval.h)
# ---------------------------------------------------------------------------------------------

_ENC = ("ln1.g", "ln1.b", "wqkv", "bqkv", "wo", "bo", "ln2.g", "ln2.b", "w1", "b1", "w2", "b2")
_ITEM = ("ln1.g", "ln1.b", "wqkv", "bqkv", "wo", "bo", "ln2.g", "ln2.b", "wq", "bq", "wo2", "bo2",
         "ln3.g", "ln3.b", "w1", "b1", "w2", "b2")


def param_names(n_layers: int, vocab: int) -> List[str]:
    names: List[str] = []
    names += [f"ctx.{l}.{p}" for l in range(n_layers) for p in _ENC]
    names += ["ctx.lnf.g", "ctx.lnf.b"]
    names += [f"ctx.kv.{l}.{p}" for l in range(n_layers) for p in ("wk", "bk", "wv", "bv")]
    names += [f"item.{l}.{p}" for l in range(n_layers) for p in _ITEM]
    names += ["item.lnf.g", "item.lnf.b"]
    names += [f"seq.{l}.{p}" for l in range(n_layers) for p in _ENC]
    names += ["seq.lnf.g", "seq.lnf.b"]
    names += [f"cross.{l}.{p}" for l in range(n_layers) for p in _ENC]
    names += ["cross.lnf.g", "cross.lnf.b"]
    names += ["cls", "pos", "head.w", "head.b"]
    if vocab:
        names.append("emb")
    return names


def pack_params(params: Dict[str, np.ndarray], n_layers: int, vocab: int) -> np.ndarray:
    """Flat float32 array of every parameter in fe_model_create order."""
    return np.concatenate([np.ascontiguousarray(params[n], dtype=np.float32).reshape(-1)
                           for n in param_names(n_layers, vocab)])


# ---------------------------------------------------------------------------------------------
# C functions (same names as the ABI)
# ---------------------------------------------------------------------------------------------

def fe_param_count(cfg: fe_config) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_param_count(ctypes.byref(cfg), ctypes.byref(n)), "fe_param_count")
    return n.value


def fe_model_create(cfg: fe_config, flat: np.ndarray) -> int:
    flat = np.ascontiguousarray(flat, dtype=np.float32)
    h = ctypes.c_void_p()
    _check(load_library().fe_model_create(ctypes.byref(cfg), flat.ctypes.data, flat.size, ctypes.byref(h)),
           "fe_model_create")
    return h.value


def fe_model_destroy(model: int) -> None:
    load_library().fe_model_destroy(model)


def fe_workspace_size(model: int, B: int, T: int, M: int, K: int, L: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_workspace_size(model, B, T, M, K, L, ctypes.byref(n)), "fe_workspace_size")
    return n.value


def fe_kv_size(model: int, B: int, T: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_kv_size(model, B, T, ctypes.byref(n)), "fe_kv_size")
    return n.value


def fe_read_device_status(model: int, ws, B: int, stream=None) -> np.ndarray:
    out = np.zeros(B, dtype=np.int32)
    _check(load_library().fe_read_device_status(model, _ptr(ws), B, _stream(stream), out.ctypes.data),
           "fe_read_device_status")
    return out


def fe_encode_context(model: int, B: int, T: int, x, ctx_ids, kv, ws, stream=None) -> None:
    _check(load_library().fe_encode_context(model, B, T, _ptr(x), _ptr(ctx_ids), _ptr(kv), _ptr(ws),
                                            ws.numel() * ws.element_size(), _stream(stream)), "fe_encode_context")


def fe_encode_items(model: int, B: int, M: int, pool, lists, K: int, L: int, kv, T: int, uniq, n_uniq, slot, H, ws,
                    stream=None) -> None:
    _check(load_library().fe_encode_items(model, B, M, _ptr(pool), _ptr(lists), K, L, _ptr(kv), T, _ptr(uniq),
                                          _ptr(n_uniq), _ptr(slot), _ptr(H), _ptr(ws),
                                          ws.numel() * ws.element_size(), _stream(stream)), "fe_encode_items")


def fe_assemble(model: int, B: int, K: int, L: int, U_cap: int, slot, H, seq, stream=None) -> None:
    _check(load_library().fe_assemble(model, B, K, L, U_cap, _ptr(slot), _ptr(H), _ptr(seq), _stream(stream)),
           "fe_assemble")


def fe_cross_sequence(model: int, B: int, K: int, L: int, seq, Cp, ws, stream=None) -> None:
    _check(load_library().fe_cross_sequence(model, B, K, L, _ptr(seq), _ptr(Cp), _ptr(ws),
                                            ws.numel() * ws.element_size(), _stream(stream)), "fe_cross_sequence")


FE_NOALLOC_SCRATCH_BYTES = 32 << 20


def fe_executor_create(model: int, n_streams: int) -> int:
    out = ctypes.c_void_p()
    _check(load_library().fe_executor_create(model, n_streams, ctypes.byref(out)), "fe_executor_create")
    return out.value


def fe_executor_submit(ex: int, B: int, T: int, M: int, K: int, L: int, x, ctx_ids, pool, lists, kv, uniq, n_uniq,
                       slot, H, seq, Cp, scores, best, ws, stream=None) -> None:
    a = fe_pass_args(B, T, M, K, L, _ptr(x), _ptr(ctx_ids), _ptr(pool), _ptr(lists), _ptr(kv), _ptr(uniq),
                     _ptr(n_uniq), _ptr(slot), _ptr(H), _ptr(seq), _ptr(Cp), _ptr(scores), _ptr(best), _ptr(ws),
                     ws.numel() * ws.element_size())
    _check(load_library().fe_executor_submit(ex, ctypes.byref(a), _stream(stream)), "fe_executor_submit")


def fe_executor_join(ex: int, stream=None) -> None:
    _check(load_library().fe_executor_join(ex, _stream(stream)), "fe_executor_join")


def fe_executor_destroy(ex: int) -> None:
    load_library().fe_executor_destroy(ex)


def fe_cross_sequence_noalloc(model: int, B: int, K: int, L: int, seq, Cp, stream=None) -> None:
    """fe_cross_sequence with the library's static scratch instead of a workspace (allocates nothing)."""
    _check(load_library().fe_cross_sequence_noalloc(model, B, K, L, _ptr(seq), _ptr(Cp), _stream(stream)),
           "fe_cross_sequence_noalloc")


def fe_score_select(model: int, B: int, K: int, Cp, scores, best, stream=None) -> None:
    _check(load_library().fe_score_select(model, B, K, _ptr(Cp), _ptr(scores), _ptr(best), _stream(stream)),
           "fe_score_select")


def fe_encode_sequences(model: int, B: int, K: int, L: int, seq, C, ws, stream=None) -> None:
    _check(load_library().fe_encode_sequences(model, B, K, L, _ptr(seq), _ptr(C), _ptr(ws),
                                              ws.numel() * ws.element_size(), _stream(stream)), "fe_encode_sequences")


def fe_score_objectives(model: int, B: int, K: int, Cp, n_obj: int, head_w, head_b, fuse_w, obj_scores, scores, best,
                        stream=None) -> None:
    _check(load_library().fe_score_objectives(model, B, K, _ptr(Cp), n_obj, _ptr(head_w), _ptr(head_b), _ptr(fuse_w),
                                              _ptr(obj_scores), _ptr(scores), _ptr(best), _stream(stream)),
           "fe_score_objectives")


def fe_naive_workspace_size(model: int, B: int, T: int, M: int, K: int, L: int, token_ids: bool) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_naive_workspace_size(model, B, T, M, K, L, 1 if token_ids else 0, ctypes.byref(n)),
           "fe_naive_workspace_size")
    return n.value


def fe_evaluate_naive(model: int, B: int, T: int, M: int, K: int, L: int, x, ctx_ids, pool, lists, Cp, scores, best,
                      ws, stream=None) -> None:
    _check(load_library().fe_evaluate_naive(model, B, T, M, K, L, _ptr(x), _ptr(ctx_ids), _ptr(pool), _ptr(lists),
                                            _ptr(Cp), _ptr(scores), _ptr(best), _ptr(ws),
                                            ws.numel() * ws.element_size(), _stream(stream)), "fe_evaluate_naive")


def fe_train_workspace_size(cfg: fe_config, B: int, T: int, M: int, K: int, L: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_train_workspace_size(ctypes.byref(cfg), B, T, M, K, L, ctypes.byref(n)),
           "fe_train_workspace_size")
    return n.value


def _need(t, name: str, dtype, numel: int) -> None:
    """Argument check for tensors handed to the library as raw pointers: dtype, size, contiguity."""
    if t is None or isinstance(t, int):
        return
    if t.dtype != dtype or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of {numel} elements, got {t.dtype} "
                         f"{tuple(t.shape)}")


def fe_train_grads(cfg: fe_config, params, B: int, T: int, M: int, K: int, L: int, x, ctx_ids, pool, lists, relevant,
                   loss_kind: int, loss, scores, grads, ws, stream=None) -> None:
    import torch
    n = fe_param_count(cfg)
    _need(params, "params", torch.float32, n)
    _need(grads, "grads", torch.float32, n)
    _need(loss, "loss", torch.float32, 1)
    _need(scores, "scores", torch.float32, B * K)
    _need(x, "x", torch.float32, B * T * cfg.d)
    _need(pool, "pool", torch.float32, B * M * cfg.d)
    _need(ctx_ids, "ctx_ids", torch.int32, B * T)
    _need(lists, "lists", torch.int32, B * K * L)
    _need(relevant, "relevant", torch.int32, B * M)
    _check(load_library().fe_train_grads(ctypes.byref(cfg), _ptr(params), B, T, M, K, L, _ptr(x), _ptr(ctx_ids),
                                         _ptr(pool), _ptr(lists), _ptr(relevant), loss_kind, _ptr(loss), _ptr(scores),
                                         _ptr(grads), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "fe_train_grads")


def fe_cache_append(args: fe_append_args, stream=None) -> None:
    st = load_library().fe_cache_append(args, _stream(stream))
    if st != FE_OK:
        _check(st, "fe_cache_append")


def fe_prefix_workspace_size(args: fe_prefix_args, grad: bool = False) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_prefix_workspace_size(ctypes.byref(args), 1 if grad else 0, ctypes.byref(n)),
           "fe_prefix_workspace_size")
    return n.value


def fe_prefix_attention(args: fe_prefix_args, stream=None) -> None:
    st = load_library().fe_prefix_attention(args, _stream(stream))
    if st != FE_OK:
        _check(st, "fe_prefix_attention")


def fe_prefix_attention_grad(args: fe_prefix_args, grads: fe_prefix_grads, stream=None) -> None:
    _check(load_library().fe_prefix_attention_grad(ctypes.byref(args), ctypes.byref(grads), _stream(stream)),
           "fe_prefix_attention_grad")


def fe_packed_page_bytes(page_rows: int, n_kv_heads: int, dh: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_packed_page_bytes(page_rows, n_kv_heads, dh, ctypes.byref(n)), "fe_packed_page_bytes")
    return n.value


def fe_packed_append(args: fe_packed_append_args, stream=None) -> None:
    st = load_library().fe_packed_append(args, _stream(stream))
    if st != FE_OK:
        _check(st, "fe_packed_append")


def fe_packed_read(args: fe_packed_read_args, stream=None) -> None:
    st = load_library().fe_packed_read(args, _stream(stream))
    if st != FE_OK:
        _check(st, "fe_packed_read")


def fe_packed_workspace_size(args: fe_packed_args, weights: bool = False) -> int:
    n = ctypes.c_size_t()
    _check(load_library().fe_packed_workspace_size(ctypes.byref(args), 1 if weights else 0, ctypes.byref(n)),
           "fe_packed_workspace_size")
    return n.value


def fe_packed_attention(args: fe_packed_args, stream=None) -> None:
    st = load_library().fe_packed_attention(args, _stream(stream))
    if st != FE_OK:
        _check(st, "fe_packed_attention")


def fe_packed_weights(args: fe_packed_args, stream=None) -> None:
    st = load_library().fe_packed_weights(args, _stream(stream))
    if st != FE_OK:
        _check(st, "fe_packed_weights")


def fe_packed_weights_strided(args: fe_packed_args, lse_ld, stream=None) -> None:
    """lse_ld: elements from one request, list, row and head to the next."""
    st = load_library().fe_packed_weights_strided(args, (ctypes.c_int64 * 4)(*lse_ld), _stream(stream))
    if st != FE_OK:
        _check(st, "fe_packed_weights_strided")


def fe_packed_evict(args: fe_packed_evict_args, stream=None) -> None:
    st = load_library().fe_packed_evict(args, _stream(stream))
    if st != FE_OK:
        _check(st, "fe_packed_evict")


def fe_trace_enable(on: bool) -> None:
    _check(load_library().fe_trace_enable(1 if on else 0), "fe_trace_enable")


def fe_trace_read_launches(capacity: int = 1 << 16) -> List[Tuple[str, float]]:
    """Recorded launches in enqueue order: (family name, kernel ms) each; consumes the records."""
    lib = load_library()
    fam = np.zeros(capacity, dtype=np.int32)
    ms = np.zeros(capacity, dtype=np.float64)
    n = ctypes.c_int64(0)
    _check(lib.fe_trace_read_launches(fam.ctypes.data, ms.ctypes.data, capacity, ctypes.byref(n)),
           "fe_trace_read_launches")
    return [(lib.fe_trace_family(int(fam[i])).decode(), float(ms[i])) for i in range(n.value)]


def fe_trace_read() -> Dict[str, Tuple[float, int]]:
    """{family: (summed kernel ms, launches)} since the last read; synchronises the traced events."""
    ms = np.zeros(FE_TRACE_FAMILIES, dtype=np.float64)
    n = np.zeros(FE_TRACE_FAMILIES, dtype=np.int64)
    lib = load_library()
    _check(lib.fe_trace_read(ms.ctypes.data, n.ctypes.data), "fe_trace_read")
    return {lib.fe_trace_family(i).decode(): (float(ms[i]), int(n[i])) for i in range(FE_TRACE_FAMILIES)}


# ---------------------------------------------------------------------------------------------
# Convenience: one model plus the buffers of one batch shape
# ---------------------------------------------------------------------------------------------

class Evaluator:
    """Owns a model handle and, per batch shape, the device buffers of the five calls.

    `params` maps the parameter names of `param_names` to float arrays; `dtype` is "f32" or
    "bf16".  All tensors are allocated with torch on the current device.
    """

    def __init__(self, d: int, n_heads: int, n_layers: int, ffn_dim: int, max_L: int, vocab: int, dtype: str,
                 params: Dict[str, np.ndarray], attention: str = "softmax"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("Evaluator needs a HIP device")
        if attention not in ("softmax", "linear"):
            raise ValueError(f"attention must be 'softmax' or 'linear', got {attention!r}")
        self.cfg = fe_config(d, n_heads, n_layers, ffn_dim, max_L, vocab, FE_BF16 if dtype == "bf16" else FE_F32,
                             FE_ATTN_LINEAR if attention == "linear" else FE_ATTN_SOFTMAX)
        self.d, self.n_layers, self.vocab, self.n_heads = d, n_layers, vocab, n_heads
        self.attention = attention
        self.act = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.handle = fe_model_create(self.cfg, pack_params(params, n_layers, vocab))
        self.buffers = None
        self.naive_buffers = None

    def close(self) -> None:
        if self.handle:
            fe_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def allocate(self, B: int, T: int, M: int, K: int, L: int) -> Dict:
        import torch
        dev = torch.device("cuda", torch.cuda.current_device())
        d, n = self.d, self.n_layers
        U_cap = min(M, K * L)
        ws_bytes = fe_workspace_size(self.handle, B, T, M, K, L)
        i32 = torch.int32
        self.buffers = dict(
            shape=(B, T, M, K, L), U_cap=U_cap,
            kv=self._kv_tensor(B, T, dev),
            uniq=torch.empty((B, U_cap), dtype=i32, device=dev),
            n_uniq=torch.empty((B,), dtype=i32, device=dev),
            slot=torch.empty((B, K, L), dtype=i32, device=dev),
            H=torch.empty((B, U_cap, d), dtype=self.act, device=dev),
            seq=torch.empty((B, K, L + 1, d), dtype=self.act, device=dev),
            Cp=torch.empty((B, K, d), dtype=torch.float32, device=dev),
            scores=torch.empty((B, K), dtype=torch.float32, device=dev),
            best=torch.empty((B,), dtype=i32, device=dev),
            ws=torch.empty((ws_bytes,), dtype=torch.uint8, device=dev),
        )
        return self.buffers

    def _kv_tensor(self, B: int, T: int, dev):
        """fe_encode_context's output: keys/values [n][2][B][T][d] act, or on linear-attention
        models the per-head state [n][B][H][dh+1][dh] fp32 (fe_kv_size bytes either way)."""
        import torch
        n, d, H = self.n_layers, self.d, self.n_heads
        if self.attention == "linear":
            shape, dt = (n, B, H, d // H + 1, d // H), torch.float32
        else:
            shape, dt = (n, 2, B, T, d), self.act
        t = torch.empty(shape, dtype=dt, device=dev)
        assert t.numel() * t.element_size() == fe_kv_size(self.handle, B, T)
        return t

    def run(self, x=None, ctx_ids=None, pool=None, lists=None, stream=None, buffers=None) -> Dict:
        """Enqueue the five calls on device tensors already resident on the GPU (into `buffers`, a
        dict from `allocate`, else the last allocated set)."""
        b = self.buffers if buffers is None else buffers
        B, T, M, K, L = b["shape"]
        h = self.handle
        fe_encode_context(h, B, T, x, ctx_ids, b["kv"], b["ws"], stream)
        fe_encode_items(h, B, M, pool, lists, K, L, b["kv"], T, b["uniq"], b["n_uniq"], b["slot"], b["H"], b["ws"],
                        stream)
        fe_assemble(h, B, K, L, b["U_cap"], b["slot"], b["H"], b["seq"], stream)
        fe_cross_sequence(h, B, K, L, b["seq"], b["Cp"], b["ws"], stream)
        fe_score_select(h, B, K, b["Cp"], b["scores"], b["best"], stream)
        return b

    def allocate_naive(self, B: int, T: int, M: int, K: int, L: int, token_ids: bool) -> Dict:
        """Outputs and workspace of the candidate-factorised baseline (fe_evaluate_naive)."""
        import torch
        dev = torch.device("cuda", torch.cuda.current_device())
        ws_bytes = fe_naive_workspace_size(self.handle, B, T, M, K, L, token_ids)
        self.naive_buffers = dict(
            shape=(B, T, M, K, L),
            Cp=torch.empty((B, K, self.d), dtype=torch.float32, device=dev),
            scores=torch.empty((B, K), dtype=torch.float32, device=dev),
            best=torch.empty((B,), dtype=torch.int32, device=dev),
            ws=torch.empty((ws_bytes,), dtype=torch.uint8, device=dev),
        )
        return self.naive_buffers

    def run_naive(self, x=None, ctx_ids=None, pool=None, lists=None, stream=None) -> Dict:
        """Enqueue the candidate-factorised evaluator (no reuse) on resident device tensors."""
        b = self.naive_buffers
        B, T, M, K, L = b["shape"]
        fe_evaluate_naive(self.handle, B, T, M, K, L, x, ctx_ids, pool, lists, b["Cp"], b["scores"], b["best"],
                          b["ws"], stream)
        return b


class Executor:
    """Whole passes of independent batches, round-robin over `n_streams` HIP streams of the
    library (fe_executor_*).  Give every stream its own buffer set (`Evaluator.allocate`): pass i
    writes set i mod n_streams, so a set is reused only after n_streams - 1 other passes."""

    def __init__(self, evaluator: "Evaluator", n_streams: int):
        self.evaluator = evaluator
        self.n_streams = n_streams
        self.handle = fe_executor_create(evaluator.handle, n_streams)

    def submit(self, buffers: Dict, x=None, ctx_ids=None, pool=None, lists=None, stream=None) -> Dict:
        """Enqueue one pass into `buffers` after the work already on `stream` (the inputs')."""
        b = buffers
        B, T, M, K, L = b["shape"]
        fe_executor_submit(self.handle, B, T, M, K, L, x, ctx_ids, pool, lists, b["kv"], b["uniq"], b["n_uniq"],
                           b["slot"], b["H"], b["seq"], b["Cp"], b["scores"], b["best"], b["ws"], stream)
        return b

    def join(self, stream=None) -> None:
        """Make `stream` wait for every submitted pass."""
        fe_executor_join(self.handle, stream)

    def close(self) -> None:
        if self.handle:
            fe_executor_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------------------------
# Lists over a shared context: paged cache and attention (include/flasheval_prefix.h)
# ---------------------------------------------------------------------------------------------

def _act(dtype: str):
    import torch
    if dtype not in ("bf16", "f32"):
        raise ValueError(f"dtype must be 'bf16' or 'f32', got {dtype!r}")
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _row_stride(t, name: str, shape: Tuple[int, ...], dtype) -> int:
    """Elements from one row to the next of a tensor [..][heads][dh] whose rows are evenly spaced and dense inside
    (column blocks of a wider tensor qualify); raises ValueError for any other layout, shape or type."""
    if t.dtype != dtype or tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected a {dtype} tensor {shape}, got {t.dtype} {tuple(t.shape)}")
    st, width = t.stride(), shape[-1] * shape[-2]
    if t.numel() == 0:
        return width
    ok = st[-1] == 1 and (shape[-2] == 1 or st[-2] == shape[-1])
    ld, rows = None, 1                      # stride of the innermost row axis longer than 1; rows inside the axis at hand
    for n, s in zip(reversed(shape[:-2]), reversed(st[:-2])):
        if n > 1:
            if ld is None:
                ld = s
            ok = ok and s == ld * rows
            rows *= n
    ld = width if ld is None else ld
    if not ok or ld < width:
        raise ValueError(f"{name}: rows of {width} elements must be dense and evenly spaced, got strides {tuple(st)} for shape "
                         f"{shape}")
    if ld > 2 ** 31 - 1:
        raise ValueError(f"{name}: a row stride of {ld} elements does not fit int32")
    return ld


class _Layouts:
    """The layout checks of one object's tensors, remembered by shapes, strides and types: a serving loop passes the same
    layouts again and again.  Prompts of ever new lengths do not: the MOST last learnt are kept."""

    MOST = 256

    def __init__(self):
        self.known = {}

    def of(self, check, *tensors):
        """What check(*tensors) returned for tensors of these layouts (it raises for those that do not fit)."""
        key = tuple([None if t is None else (t.shape, t.stride(), t.dtype) for t in tensors])
        got = self.known.get(key)
        if got is None:
            got = check(*tensors)
            if len(self.known) >= self.MOST:
                self.known.pop(list(self.known)[0], None)        # the oldest; another thread may have been here
            self.known[key] = got
        return got


def _on_device(tensors) -> int:
    """Index of the current HIP device, on which all the tensors have to be."""
    import torch
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and (t.get_device() != index or index < 0):
            raise ValueError(f"every tensor must be on the current HIP device, got one on {t.device}")
    if torch.cuda.current_device() != index:
        raise ValueError(f"the tensors are on device {index}, the current HIP device is {torch.cuda.current_device()}")
    return index


def _stream_on(index: int, stream) -> int:
    return _current_stream(index) if stream is None else _stream(stream)


def _allocated_for(stream, *tensors, home=None) -> None:
    """Tensors allocated on the stream `home` (the current one) that `stream`, another one, is about to use: it waits for what
    `home` still does in their memory, and the memory is not given out again before its own work there has ended."""
    import torch
    home = torch.cuda.current_stream() if home is None else home
    if stream is None or _stream(stream) == home.cuda_stream:
        return
    other = torch.cuda.ExternalStream(_stream(stream)) if _stream(stream) else torch.cuda.default_stream()
    other.wait_stream(home)
    for t in tensors:
        if t is not None:
            t.record_stream(other)


class _Kept:
    """Tensors that an object allocates for itself, on the current stream, and keeps: handed once to every other stream that
    uses them."""

    def __init__(self, *tensors):
        import torch
        self.tensors, self.home = tensors, torch.cuda.current_stream()
        self.known = {self.home.cuda_stream}

    def use_on(self, handle: int) -> None:
        if handle in self.known:
            return
        import torch
        capturing = torch.cuda.is_current_stream_capturing()
        if capturing and torch.cuda.current_stream().cuda_stream != self.home.cuda_stream:
            return                           # a capture cannot wait for work outside it; it begins after that
        _allocated_for(handle, *self.tensors, home=self.home)
        if not capturing:
            self.known.add(handle)           # last: another thread that finds it there need not wait


def _addr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class PagedCache:
    """Keys and values of N growing sequences in pages of a shared pool (fe_cache_append).

    k_pages, v_pages [n_pages][page_rows][n_kv_heads][dh] and table [N][cols] int32 are the caller's:
    table[s][c] names the page that holds rows c * page_rows .. of sequence s.  len [N] int32 counts the rows
    of every sequence and is advanced by `append`."""

    def __init__(self, k_pages, v_pages, table, length=None):
        import torch
        if k_pages.dim() != 4:
            raise ValueError(f"k_pages: expected [pages][rows][heads][dh], got {tuple(k_pages.shape)}")
        if k_pages.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"k_pages: bfloat16 or float32, got {k_pages.dtype}")
        shape = tuple(k_pages.shape)
        self.page_ld = _row_stride(k_pages, "k_pages", shape, k_pages.dtype)
        if _row_stride(v_pages, "v_pages", shape, k_pages.dtype) != self.page_ld:
            raise ValueError("k_pages and v_pages must have the same row stride")
        if table.dim() != 2:
            raise ValueError(f"table: expected [sequences][columns], got {tuple(table.shape)}")
        self.N, self.cols = table.shape
        _need(table, "table", torch.int32, self.N * self.cols)
        self.len = torch.zeros(self.N, dtype=torch.int32, device=table.device) if length is None else length
        _need(self.len, "length", torch.int32, self.N)
        self.k_pages, self.v_pages, self.table = k_pages, v_pages, table
        self.status = torch.zeros(self.N, dtype=torch.int32, device=table.device)
        _on_device((k_pages, v_pages, table, self.len))
        self._kept = _Kept(self.status, self.len if length is None else None)
        a = self.args = fe_append_args()
        a.dtype = FE_BF16 if k_pages.dtype == torch.bfloat16 else FE_F32
        a.n_pages, a.page_rows, a.n_kv_heads, a.dh = shape
        a.N, a.table_cols, a.page_ld = self.N, self.cols, self.page_ld
        a.k_pages, a.v_pages, a.table = _ptr(k_pages), _ptr(v_pages), _ptr(table)
        a.len, a.status = _ptr(self.len), _ptr(self.status)
        self._layouts = _Layouts()

    def _check(self, k, v, q, q_out, freq, new_len, pos0, len_out):
        """(rows, n_heads, k_ld, v_ld, q_ld, q_out_ld, rot) of an append's tensors."""
        import torch
        hkv, dh, dt, N = self.k_pages.shape[2], self.k_pages.shape[3], self.k_pages.dtype, self.N
        if k.dim() != 4:
            raise ValueError(f"k: expected [sequences][rows][heads][dh], got {tuple(k.shape)}")
        S = k.shape[1]
        k_ld, v_ld = (_row_stride(t, n, (N, S, hkv, dh), dt) for t, n in ((k, "k"), (v, "v")))
        H = q_ld = q_out_ld = 0
        if q is not None:
            if q.dim() != 4:
                raise ValueError(f"q: expected [sequences][rows][heads][dh], got {tuple(q.shape)}")
            H = q.shape[2]
            q_ld, q_out_ld = (_row_stride(t, n, (N, S, H, dh), dt) for t, n in ((q, "q"), (q_out, "q_out")))
        if freq is not None:
            _need(freq, "freq", torch.float64, freq.numel())
        for t, name in ((new_len, "new_len"), (pos0, "pos0"), (len_out, "len_out")):
            _need(t, name, torch.int32, N)
        return S, H, k_ld, v_ld, q_ld, q_out_ld, 0 if freq is None else 2 * freq.numel()

    def append(self, k, v, q=None, q_out=None, new_len=None, pos0=None, freq=None, neighbours=False, len_out=None,
               stream=None):
        """Append rows k, v [N][S][n_kv_heads][dh] (the first new_len[s] of sequence s); with `freq` (float64 [rot / 2])
        keys and q [N][S][n_heads][dh] are turned by their positions pos0[s] + row.  q_out defaults to a new
        tensor; it is returned.  The lengths advance in place, or into len_out when that is given.
        `status` [N] holds FE_DEV_BAD_PAGE for a sequence with a row that found no page."""
        a = self.args
        if (q is None) != (q_out is None):
            if q is None:
                raise ValueError("q_out without q")
            q_out = q.new_empty(q.shape)
            _allocated_for(stream, q_out)
        a.S, a.n_heads, a.k_ld, a.v_ld, a.q_ld, a.q_out_ld, a.rot = self._layouts.of(
            self._check, k, v, q, q_out, freq, new_len, pos0, len_out)
        handle = _stream_on(_on_device((k, v, q, q_out, freq, new_len, pos0, len_out, self.k_pages)), stream)
        self._kept.use_on(handle)
        a.neighbours = 1 if neighbours else 0
        a.q, a.k, a.v, a.q_out, a.freq = _addr(q), k.data_ptr(), v.data_ptr(), _addr(q_out), _addr(freq)
        a.new_len, a.pos0, a.len_out = _addr(new_len), _addr(pos0), a.len if len_out is None else len_out.data_ptr()
        fe_cache_append(a, handle)
        return q_out


class PrefixAttention:
    """Attention of K lists per request over the request's shared rows and each list's own rows
    (fe_prefix_attention), with its outputs and workspace for one batch shape; `train=True` also keeps lse and allows `grad`.

    `run` takes q [B][K][S][n_heads][dh], ctx_k and ctx_v [B][T][n_kv_heads][dh] (a layer's slice of
    fe_encode_context's cache, viewed with its heads, is one), and own_k and own_v [B][K][L][n_kv_heads][dh], or
    with page_rows > 0 the pages of a PagedCache [n_pages][page_rows][n_kv_heads][dh] and `table`
    [B][K][L / page_rows] int32.  ctx_len [B], q_len [B][K] and own_len [B][K] int32 give the rows in use.  The outputs
    belong to this object and are overwritten by its next call, as is its workspace: one object per stream.  The calls work outside
    torch's autograd, whatever their tensors require: `run` returns no history, and what `grad` returns is handed on with
    torch.autograd.backward((q, ctx_k, ctx_v, own_k, own_v), grads)."""

    def __init__(self, B: int, K: int, S: int, T: int, L: int, n_heads: int, n_kv_heads: int, dh: int, dtype: str,
                 causal: bool = False, scale: Optional[float] = None, page_rows: int = 0, n_pages: int = 0,
                 train: bool = False):
        self.act, self.train = _act(dtype), train
        a = self.args = fe_prefix_args()
        a.dtype = FE_BF16 if dtype == "bf16" else FE_F32
        a.B, a.K, a.S, a.T, a.L, a.n_heads, a.n_kv_heads, a.dh = B, K, S, T, L, n_heads, n_kv_heads, dh
        a.page_rows, a.n_pages, a.causal = page_rows, n_pages, 1 if causal else 0
        a.scale = dh ** -0.5 if scale is None else scale
        self.ws_bytes = fe_prefix_workspace_size(a)
        if train:
            self.ws_bytes = max(self.ws_bytes, fe_prefix_workspace_size(a, True))
        self.out = None
        self.grads = None
        self.q_shape, self.ctx_shape = (B, K, S, n_heads, dh), (B, T, n_kv_heads, dh)
        self.own_shape = (n_pages, page_rows, n_kv_heads, dh) if page_rows else (B, K, L, n_kv_heads, dh)
        self._layouts = _Layouts()

    def allocate(self):
        """Outputs and workspace on the current device and stream (done by the first `run`)."""
        import torch
        a, dev = self.args, torch.device("cuda", torch.cuda.current_device())
        self.out = torch.empty((a.B, a.K, a.S, a.n_heads, a.dh), dtype=self.act, device=dev)
        self.lse = torch.empty((a.B, a.K, a.S, a.n_heads), dtype=torch.float32, device=dev) if self.train else None
        rest = self.train and self.act == torch.bfloat16
        self.out_rest = torch.empty(self.q_shape, dtype=torch.int8, device=dev) if rest else None
        self.ws = torch.empty(max(16, self.ws_bytes), dtype=torch.uint8, device=dev)
        a.out, a.lse, a.out_rest = _ptr(self.out), _ptr(self.lse), _ptr(self.out_rest)
        a.ws, a.ws_bytes = _ptr(self.ws), self.ws_bytes
        a.out_ld = a.n_heads * a.dh
        if self.train:
            self.grads = (torch.empty_like(self.out),
                          *(torch.empty((a.B, a.T, a.n_kv_heads, a.dh), dtype=self.act, device=dev) for _ in range(2)),
                          *(torch.empty((a.B, a.K, a.L, a.n_kv_heads, a.dh), dtype=self.act, device=dev) for _ in range(2)))
        self._kept = _Kept(self.out, self.lse, self.out_rest, self.ws, *(self.grads or ()))

    def _check(self, q, ctx_k, ctx_v, own_k, own_v, table, ctx_len, own_len, q_len):
        """(q_ld, ctx_ld, own_ld) of a call's tensors."""
        import torch
        a, act, i32 = self.args, self.act, torch.int32
        q_ld, lds = _row_stride(q, "q", self.q_shape, act), []
        for k, v, name, shape, n in ((ctx_k, ctx_v, "ctx", self.ctx_shape, a.T), (own_k, own_v, "own", self.own_shape, a.L)):
            if n and (k is None or v is None):
                raise ValueError(f"{name}_k, {name}_v: missing")
            ld = [_row_stride(t, f"{name}_{x}", shape, act) if n else 0 for t, x in ((k, "k"), (v, "v"))]
            if ld[0] != ld[1]:
                raise ValueError(f"{name}_k and {name}_v must have the same row stride")
            lds.append(ld[0])
        if (table is None) != (a.page_rows == 0):
            raise ValueError("a table and page_rows > 0 go together")
        if table is not None:
            _need(table, "table", i32, a.B * a.K * (a.L // a.page_rows))
        _need(ctx_len, "ctx_len", i32, a.B)
        _need(q_len, "q_len", i32, a.B * a.K)
        _need(own_len, "own_len", i32, a.B * a.K)
        return q_ld, lds[0], lds[1]

    def _take(self, stream, *tensors):
        a = self.args
        q, ctx_k, ctx_v, own_k, own_v, table, ctx_len, own_len, q_len = tensors
        a.q_ld, a.ctx_ld, a.own_ld = self._layouts.of(self._check, *tensors)
        index = _on_device(tensors)
        if self.out is None:
            self.allocate()
        elif self.out.get_device() != index:
            raise ValueError(f"the outputs are on {self.out.device}, the tensors on device {index}")
        a.q, a.ctx_k, a.ctx_v, a.own_k, a.own_v = q.data_ptr(), _addr(ctx_k), _addr(ctx_v), _addr(own_k), _addr(own_v)
        a.table, a.ctx_len, a.own_len, a.q_len = _addr(table), _addr(ctx_len), _addr(own_len), _addr(q_len)
        handle = _stream_on(index, stream)
        self._kept.use_on(handle)
        return handle

    def run(self, q, ctx_k, ctx_v, own_k, own_v, table=None, ctx_len=None, own_len=None, q_len=None, stream=None):
        """Enqueue the attention; returns out [B][K][S][n_heads][dh] (self.lse holds the log sums when training)."""
        handle = self._take(stream, q, ctx_k, ctx_v, own_k, own_v, table, ctx_len, own_len, q_len)
        fe_prefix_attention(self.args, handle)
        return self.out

    def grad(self, dout, q, ctx_k, ctx_v, own_k, own_v, table=None, ctx_len=None, own_len=None, q_len=None, stream=None):
        """Gradients (dq, dctx_k, dctx_v, down_k, down_v) of the last `run`, which must have had the same tensors."""
        if not self.train:
            raise ValueError("grad needs train=True")
        if self.out is None:
            raise ValueError("grad follows run")
        handle = self._take(stream, q, ctx_k, ctx_v, own_k, own_v, table, ctx_len, own_len, q_len)
        a, g = self.args, fe_prefix_grads()
        g.dout_ld = self._layouts.of(lambda t: _row_stride(t, "dout", self.q_shape, self.act), dout)
        _on_device((dout, q))
        g.dout = dout.data_ptr()
        g.dq_ld, g.dctx_ld, g.down_ld = a.n_heads * a.dh, a.n_kv_heads * a.dh, a.n_kv_heads * a.dh
        g.dq, g.dctx_k, g.dctx_v, g.down_k, g.down_v = (t.data_ptr() for t in self.grads)
        fe_prefix_attention_grad(a, g, handle)
        return self.grads


# ---------------------------------------------------------------------------------------------
# A cache in 4 bits (include/flasheval_packed.h)
# ---------------------------------------------------------------------------------------------

class PagedCache4:
    """Keys and values of N growing sequences in 4 bits, in pages of a shared pool (fe_packed_append and its kin).

    pages [n_pages][page_bytes(page_rows, n_kv_heads, dh)] uint8 and table [N][cols] int32 are the caller's:
    table[s][c] names the page that holds rows c * page_rows .. of sequence s.  len [N] int32 counts the rows
    of every sequence; `append` advances it, `evict` sets that of the cache it fills.  A shared context is such a cache of B
    sequences, the lists' own rows one of B * K; both may use one pool.  Several threads may call one cache: every call has
    arguments of its own.  `status` is that of the last append or eviction."""

    def __init__(self, pages, table, page_rows: int, n_kv_heads: int, dh: int, length=None):
        import torch
        width = self.page_bytes(page_rows, n_kv_heads, dh)
        if pages.dtype != torch.uint8 or pages.dim() != 2 or pages.shape[1] != width or pages.stride(1) != 1:
            raise ValueError(f"pages: expected a uint8 tensor [pages][{width}] with dense rows, got {pages.dtype} "
                             f"{tuple(pages.shape)}")
        if table.dim() != 2:
            raise ValueError(f"table: expected [sequences][columns], got {tuple(table.shape)}")
        self.N, self.cols = table.shape
        _need(table, "table", torch.int32, self.N * self.cols)
        self.len = torch.zeros(self.N, dtype=torch.int32, device=table.device) if length is None else length
        _need(self.len, "length", torch.int32, self.N)
        self.pages, self.table, self.page_rows, self.n_kv_heads, self.dh = pages, table, page_rows, n_kv_heads, dh
        self.capacity = self.cols * page_rows
        self.status = torch.zeros(self.N, dtype=torch.int32, device=table.device)
        _on_device((pages, table, self.len))
        self._kept = _Kept(self.status, self.len if length is None else None)
        c = self.cache = fe_packed_cache(_ptr(pages), pages.stride(0) if pages.shape[0] > 1 else width, _ptr(table),
                                         _ptr(self.len), self.N, self.cols, page_rows, pages.shape[0])
        self.args, self.read_args, self.evict_args = (t() for t in (fe_packed_append_args, fe_packed_read_args,
                                                                    fe_packed_evict_args))
        self.args.cache = self.read_args.cache = self.evict_args.from_ = c
        for a in (self.args, self.read_args, self.evict_args):
            a.n_kv_heads, a.dh = n_kv_heads, dh
        self.args.status = self.evict_args.status = _ptr(self.status)
        self._layouts, self._read_layouts = _Layouts(), _Layouts()

    @staticmethod
    def page_bytes(page_rows: int, n_kv_heads: int, dh: int) -> int:
        """Bytes of a page: 17/32 of a byte for a column of keys and one of values, heads rounded up to 16 bytes."""
        return fe_packed_page_bytes(page_rows, n_kv_heads, dh)

    def _type(self, t, name: str):
        import torch
        if t.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"{name}: bfloat16 or float32, got {t.dtype}")
        return FE_BF16 if t.dtype == torch.bfloat16 else FE_F32

    def _check(self, k, v, q, q_out, freq, new_len, pos0, len_out):
        """(dtype, rows, n_heads, k_ld, v_ld, q_ld, q_out_ld, rot) of an append's tensors."""
        import torch
        act, N = self._type(k, "k"), self.N
        if k.dim() != 4:
            raise ValueError(f"k: expected [sequences][rows][heads][dh], got {tuple(k.shape)}")
        S, dt = k.shape[1], k.dtype
        k_ld, v_ld = (_row_stride(t, n, (N, S, self.n_kv_heads, self.dh), dt) for t, n in ((k, "k"), (v, "v")))
        H = q_ld = q_out_ld = 0
        if q is not None:
            if q.dim() != 4:
                raise ValueError(f"q: expected [sequences][rows][heads][dh], got {tuple(q.shape)}")
            H = q.shape[2]
            q_ld, q_out_ld = (_row_stride(t, n, (N, S, H, self.dh), dt) for t, n in ((q, "q"), (q_out, "q_out")))
        if freq is not None:
            _need(freq, "freq", torch.float64, freq.numel())
        for t, name in ((new_len, "new_len"), (pos0, "pos0"), (len_out, "len_out")):
            _need(t, name, torch.int32, N)
        return act, S, H, k_ld, v_ld, q_ld, q_out_ld, 0 if freq is None else 2 * freq.numel()

    def append(self, k, v, q=None, q_out=None, new_len=None, pos0=None, freq=None, neighbours=False, len_out=None,
               stream=None):
        """Append rows k, v [N][S][n_kv_heads][dh], bf16 or fp32 (the first new_len[s] of sequence s); with `freq` (float64
        [rot / 2]) keys and q [N][S][n_heads][dh] are turned by their positions pos0[s] + row.  q_out defaults to a new
        tensor and may not be q; it is returned.  The lengths advance in place, or into len_out when that is given.
        `status` [N] holds FE_DEV_BAD_PAGE for a sequence with a row that found no page."""
        a = fe_packed_append_args.from_buffer_copy(self.args)
        if (q is None) != (q_out is None):
            if q is None:
                raise ValueError("q_out without q")
            q_out = q.new_empty(q.shape)
            _allocated_for(stream, q_out)
        a.dtype, a.S, a.n_heads, a.k_ld, a.v_ld, a.q_ld, a.q_out_ld, a.rot = self._layouts.of(
            self._check, k, v, q, q_out, freq, new_len, pos0, len_out)
        handle = _stream_on(_on_device((k, v, q, q_out, freq, new_len, pos0, len_out, self.pages)), stream)
        self._kept.use_on(handle)
        a.neighbours = 1 if neighbours else 0
        a.q, a.k, a.v, a.q_out, a.freq = _addr(q), k.data_ptr(), v.data_ptr(), _addr(q_out), _addr(freq)
        a.new_len, a.pos0, a.len_out = _addr(new_len), _addr(pos0), a.cache.len if len_out is None else len_out.data_ptr()
        fe_packed_append(a, handle)
        return q_out

    def _check_read(self, k, v, start, count):
        """(dtype, rows, k_ld, v_ld) of a read's tensors."""
        import torch
        t = v if k is None else k
        act = self._type(t, "k")
        if t.dim() != 4:
            raise ValueError(f"k, v: expected [sequences][rows][heads][dh], got {tuple(t.shape)}")
        shape = (self.N, t.shape[1], self.n_kv_heads, self.dh)
        lds = [0 if x is None else _row_stride(x, n, shape, t.dtype) for x, n in ((k, "k"), (v, "v"))]
        _need(start, "start", torch.int32, self.N)
        _need(count, "count", torch.int32, self.N)
        return act, t.shape[1], lds[0], lds[1]

    def read(self, k=None, v=None, start=None, count=None, stream=None):
        """The values that rows start[s] .. start[s] + count[s] stand for, into k and v [N][S][n_kv_heads][dh], bf16 or
        fp32 (exact in both); either may be None.  Without `start` from row 0, without `count` up to the length; other
        rows of k and v are left as they were.  Without k and v: new bf16 tensors of the cache's capacity, zeros past the
        length.  Returns (k, v)."""
        import torch
        a = fe_packed_read_args.from_buffer_copy(self.read_args)
        if k is None and v is None:
            k, v = (torch.zeros((self.N, self.capacity, self.n_kv_heads, self.dh), dtype=torch.bfloat16,
                                device=self.pages.device) for _ in range(2))
            _allocated_for(stream, k, v)
        a.dtype, a.S, a.k_ld, a.v_ld = self._read_layouts.of(self._check_read, k, v, start, count)
        handle = _stream_on(_on_device((v if k is None else k, v, start, count, self.pages)), stream)
        self._kept.use_on(handle)
        a.k, a.v, a.start, a.count = _addr(k), _addr(v), _addr(start), _addr(count)
        fe_packed_read(a, handle)
        return k, v

    def evict(self, weights, to: "PagedCache4", keep: int, first: int = 0, recent: int = 0, weights_out=None, kept=None,
              stream=None):
        """Fill `to`, a cache of as many sequences in pages that none of this one's sequences use, with the `keep` rows of
        every sequence and key head that matter: the `first` and the `recent` ones, and of the others those of
        greatest weights [N][n_kv_heads][capacity] (fp32; of equal ones the lower index).  Sets to.len; rows keep their
        order and their bits.  Their weights go to weights_out [N][n_kv_heads][to.capacity] when given, no
        part of weights; their indices here to kept [N][n_kv_heads][keep] int32 (-1 where there are fewer), which is
        returned.  `status` holds FE_DEV_BAD_PAGE for a sequence with rows of no page."""
        import torch
        a = fe_packed_evict_args.from_buffer_copy(self.evict_args)
        if (to.N, to.n_kv_heads, to.dh) != (self.N, self.n_kv_heads, self.dh):
            raise ValueError(f"to: expected {self.N} sequences of {self.n_kv_heads} heads of {self.dh}, got "
                             f"{(to.N, to.n_kv_heads, to.dh)}")
        if kept is None:
            kept = torch.empty((self.N, self.n_kv_heads, keep), dtype=torch.int32, device=self.pages.device)
            _allocated_for(stream, kept)
        _need(weights, "weights", torch.float32, self.N * self.n_kv_heads * self.capacity)
        _need(weights_out, "weights_out", torch.float32, self.N * self.n_kv_heads * to.capacity)
        _need(kept, "kept", torch.int32, self.N * self.n_kv_heads * keep)
        handle = _stream_on(_on_device((weights, weights_out, kept, self.pages, to.pages)), stream)
        self._kept.use_on(handle)
        to._kept.use_on(handle)
        a.to, a.keep, a.first, a.recent = to.cache, keep, first, recent
        a.weight, a.weight_out, a.kept = weights.data_ptr(), _addr(weights_out), kept.data_ptr()
        fe_packed_evict(a, handle)
        return kept


class PrefixAttention4:
    """Attention of K lists per request over shared rows and each list's own rows, both held in 4 bits (fe_packed_attention),
    and the weight that every cached row received (fe_packed_weights), with outputs and workspace for one batch shape.

    `run` takes q [B][K][S][n_heads][dh], `ctx`, a PagedCache4 of B sequences with a capacity of T rows, and `own`, one of
    B * K sequences with a capacity of L rows (T = 0 or L = 0: None); their lengths are the rows in use, q_len [B][K]
    int32 the query rows in use, with `causal` the last own rows.  out and lse [B][K][S][n_heads] belong to this
    object and are overwritten by its next call, as is its workspace: one object per stream.  For answering: autograd
    records nothing here."""

    def __init__(self, B: int, K: int, S: int, T: int, L: int, n_heads: int, n_kv_heads: int, dh: int, dtype: str,
                 causal: bool = False, scale: Optional[float] = None):
        self.act, self.B, self.K, self.T, self.L = _act(dtype), B, K, T, L
        a = self.args = fe_packed_args()
        a.dtype = FE_BF16 if dtype == "bf16" else FE_F32
        a.B, a.K, a.S, a.n_heads, a.n_kv_heads, a.dh = B, K, S, n_heads, n_kv_heads, dh
        a.causal = 1 if causal else 0
        a.scale = dh ** -0.5 if scale is None else scale
        if T < 0 or L < 0:
            raise ValueError(f"T and L must be >= 0, got {T} and {L}")
        # workspaces go by the capacity, however it is cut into pages
        a.ctx = fe_packed_cache(None, 0, None, None, B if T else 0, 1, T, 1)
        a.own = fe_packed_cache(None, 0, None, None, B * K if L else 0, 1, L, 1)
        a.ctx_w, a.own_w = (1 if T else None), (1 if L else None)      # sizes only: the largest workspace
        self.ws_bytes = max(fe_packed_workspace_size(a), fe_packed_workspace_size(a, True))
        a.ctx_w = a.own_w = None
        self.q_shape, self.heads = (B, K, S, n_heads, dh), (n_kv_heads, dh)
        self.out = self.lse = None
        self._layouts = _Layouts()

    def allocate(self):
        """Outputs and workspace on the current device and stream (done by the first `run` or `weigh`)."""
        import torch
        a, dev = self.args, torch.device("cuda", torch.cuda.current_device())
        self.out = torch.empty(self.q_shape, dtype=self.act, device=dev)
        self.lse = torch.empty(self.q_shape[:-1], dtype=torch.float32, device=dev)
        self.ws = torch.empty(max(16, self.ws_bytes), dtype=torch.uint8, device=dev)
        a.ws, a.ws_bytes = _ptr(self.ws), self.ws_bytes
        a.out, a.out_ld = _ptr(self.out), a.n_heads * a.dh
        self._kept = _Kept(self.out, self.lse, self.ws)

    def _check(self, q, q_len):
        import torch
        _need(q_len, "q_len", torch.int32, self.B * self.K)
        return _row_stride(q, "q", self.q_shape, self.act)

    def _take(self, stream, q, ctx, own, q_len, *tensors):
        a = self.args
        a.q_ld = self._layouts.of(self._check, q, q_len)
        for cache, name, n, capacity in ((ctx, "ctx", self.B, self.T), (own, "own", self.B * self.K, self.L)):
            if (cache is None) != (capacity == 0):
                raise ValueError(f"{name}: a cache and a capacity above 0 go together")
            if cache is not None and ((cache.N, cache.capacity) != (n, capacity) or (cache.n_kv_heads, cache.dh) != self.heads):
                raise ValueError(f"{name}: expected {n} sequences of {capacity} rows with {self.heads[0]} heads of {self.heads[1]}, got "
                                 f"{cache.N} of {cache.capacity} with {cache.n_kv_heads} of {cache.dh}")
        index = _on_device((q, q_len, *tensors, None if ctx is None else ctx.pages, None if own is None else own.pages))
        if self.out is None:
            self.allocate()
        elif self.out.get_device() != index:
            raise ValueError(f"the outputs are on {self.out.device}, the tensors on device {index}")
        if ctx is not None:
            a.ctx = ctx.cache
        if own is not None:
            a.own = own.cache
        a.q, a.q_len = q.data_ptr(), _addr(q_len)
        handle = _stream_on(index, stream)
        for kept in (self, ctx, own):
            if kept is not None:
                kept._kept.use_on(handle)
        return handle

    def run(self, q, ctx: Optional[PagedCache4], own: Optional[PagedCache4], q_len=None, stream=None):
        """Enqueue the attention; returns out [B][K][S][n_heads][dh] (self.lse holds the log sums)."""
        handle = self._take(stream, q, ctx, own, q_len)
        self.args.lse = self.lse.data_ptr()
        fe_packed_attention(self.args, handle)
        return self.out

    def weigh(self, q, lse, ctx: Optional[PagedCache4], own: Optional[PagedCache4], ctx_w=None, own_w=None, q_len=None,
              ctx_w_out=None, own_w_out=None, stream=None):
        """Add the attention weight that every cached row received from the query rows (lse: `run`'s, or such log sums with
        any strides) to ctx_w [B][n_kv_heads][T] and own_w [B * K][n_kv_heads][L] fp32 (either may be None), in place or into
        the outputs.  Returns the two tensors written."""
        import torch
        a, Hkv = self.args, self.heads[0]
        ctx_w_out, own_w_out = (w if o is None else o for w, o in ((ctx_w, ctx_w_out), (own_w, own_w_out)))
        for t, name, n in ((ctx_w, "ctx_w", self.B * self.T), (ctx_w_out, "ctx_w_out", self.B * self.T),
                           (own_w, "own_w", self.B * self.K * self.L), (own_w_out, "own_w_out", self.B * self.K * self.L)):
            _need(t, name, torch.float32, n * Hkv)
        if lse.dtype != torch.float32 or lse.shape != self.q_shape[:-1]:
            _need(lse, "lse", torch.float32, self.B * self.K * self.q_shape[2] * self.q_shape[3])
        handle = self._take(stream, q, ctx, own, q_len, lse, ctx_w, own_w, ctx_w_out, own_w_out)
        a.lse = lse.data_ptr()
        a.ctx_w, a.own_w, a.ctx_w_out, a.own_w_out = _addr(ctx_w), _addr(own_w), _addr(ctx_w_out), _addr(own_w_out)
        if lse.is_contiguous():
            fe_packed_weights(a, handle)
        else:
            fe_packed_weights_strided(a, lse.stride(), handle)
        return ctx_w_out, own_w_out
