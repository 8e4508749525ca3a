"""ctypes binding of libeldr_moe.so: argument marshalling only.

Each function has the name and argument order of the C entry point it wraps
(see include/eldr_moe.h); torch tensors stand in for device pointers and the
stream defaults to torch's current stream.  Every step of the layer runs in
the library's HIP kernels; there is no fallback, and a missing library or a
non-zero status raises.
"""
from __future__ import annotations

import ctypes
import os
import re
from dataclasses import dataclass

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libeldr_moe.so")
INCLUDE_DIR = os.path.join(os.path.dirname(_PKG), "include")
HEADER_PATH = os.path.join(INCLUDE_DIR, "eldr_moe.h")
HEADER_PATHS = (HEADER_PATH, os.path.join(INCLUDE_DIR, "eldr_signature.h"),
                os.path.join(INCLUDE_DIR, "eldr_calibration.h"),
                os.path.join(INCLUDE_DIR, "eldr_attention.h"),
                os.path.join(INCLUDE_DIR, "eldr_kv_cache.h"),
                os.path.join(INCLUDE_DIR, "eldr_route.h"))

MOE_OK = 0
MOE_ERR_INVALID = -1
MOE_ERR_UNSUPPORTED = -2
MOE_ERR_WORKSPACE = -3
MOE_ERR_HIP = -4

# Shape limits of the layer calls (include/eldr_moe.h).
MOE_MAX_E = 256
MOE_MAX_K = 16
MOE_MAX_T = 4096
MOE_MAX_H = 16384
MOE_MAX_I = 16384


class MoeDims(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("E", ctypes.c_int32),
                ("K", ctypes.c_int32), ("I", ctypes.c_int32)]

    def __repr__(self) -> str:
        return f"MoeDims(T={self.T}, H={self.H}, E={self.E}, K={self.K}, I={self.I})"


class AttnDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("R", "Hq", "Hkv", "D", "block_size", "max_blocks",
                                              "num_blocks", "kv_type")] + [("block_stride", ctypes.c_int64)]

    def __repr__(self) -> str:
        return "AttnDims(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class MoeError(RuntimeError):
    def __init__(self, fn: str, status: int, text: str):
        super().__init__(f"{fn} returned {status}: {text}")
        self.status = status


_vp = ctypes.c_void_p
_SIGNATURES = {
    "moe_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "moe_abi_version": (ctypes.c_int, []),
    "moe_gate_topk": (ctypes.c_int, [_vp, _vp, MoeDims, _vp, _vp, _vp, _vp]),
    "moe_bucket": (ctypes.c_int, [_vp, MoeDims, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "moe_ffn_workspace_bytes": (ctypes.c_size_t, [MoeDims]),
    "moe_expert_ffn": (ctypes.c_int, [_vp] * 7 + [MoeDims, _vp, _vp, ctypes.c_size_t, _vp]),
    "moe_expert_ffn_up": (ctypes.c_int, [_vp] * 6 + [MoeDims, _vp, ctypes.c_size_t, _vp]),
    "moe_expert_ffn_noalloc": (ctypes.c_int, [_vp] * 7 + [MoeDims, _vp, _vp]),
    "moe_expert_ffn_noalloc_max_bytes": (ctypes.c_size_t, []),
    "moe_expert_ffn_up_routed": (ctypes.c_int, [_vp] * 3 + [MoeDims] + [_vp] * 7 +
                                 [ctypes.c_size_t, _vp]),
    "moe_expert_ffn_mxfp4_up_routed": (ctypes.c_int, [_vp] * 4 + [MoeDims] + [_vp] * 7 +
                                       [ctypes.c_size_t, _vp]),
    "moe_expert_ffn_routed": (ctypes.c_int, [_vp] * 4 + [MoeDims] + [_vp] * 8 +
                              [ctypes.c_size_t, _vp, _vp]),
    "moe_expert_ffn_mxfp4_routed": (ctypes.c_int, [_vp] * 6 + [MoeDims] + [_vp] * 8 +
                                    [ctypes.c_size_t, _vp, _vp]),
    "moe_ffn_sync_bytes": (ctypes.c_size_t, [MoeDims]),
    "moe_expert_ffn_down": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, MoeDims, ctypes.c_size_t,
                                           _vp, _vp]),
    "moe_combine": (ctypes.c_int, [_vp, _vp, _vp, MoeDims, _vp, _vp]),
    "moe_pack_up_weights": (ctypes.c_int, [_vp, _vp] + [ctypes.c_int32] * 3 + [_vp, _vp]),
    "moe_pack_down_weights": (ctypes.c_int, [_vp] + [ctypes.c_int32] * 3 + [_vp, _vp]),
    "moe_pack_mxfp4_up": (ctypes.c_int, [_vp, _vp, _vp, _vp, ctypes.c_int32, ctypes.c_int32,
                                         ctypes.c_int32, _vp, _vp, _vp]),
    "moe_pack_mxfp4_down": (ctypes.c_int, [_vp, _vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                           _vp, _vp, _vp]),
    "moe_expert_ffn_mxfp4": (ctypes.c_int, [_vp] * 9 + [MoeDims, _vp, _vp, ctypes.c_size_t, _vp]),
    "moe_expert_ffn_mxfp4_up": (ctypes.c_int, [_vp] * 7 + [MoeDims, _vp, ctypes.c_size_t, _vp]),
    "moe_expert_ffn_mxfp4_down": (ctypes.c_int, [_vp] * 7 + [MoeDims, ctypes.c_size_t, _vp, _vp]),
    "moe_sig_capture": (ctypes.c_int, [_vp, _vp] + [ctypes.c_int32] * 7 + [_vp, _vp, _vp]),
    "moe_sig_reset": (ctypes.c_int, [_vp] + [ctypes.c_int32] * 4 + [_vp, _vp]),
    "moe_sig_request_counts": (ctypes.c_int, [_vp, _vp, _vp] + [ctypes.c_int32] * 5 + [_vp, _vp]),
    "moe_kv_append": (ctypes.c_int, [_vp] * 3 + [ctypes.c_int64] * 3 + [ctypes.c_int32] * 2 + [_vp, ctypes.c_int32] +
                      [_vp] * 3 + [ctypes.c_int32] * 3 + [_vp, AttnDims] + [_vp] * 6),
    "moe_attn_workspace_bytes": (ctypes.c_size_t, [AttnDims]),
    "moe_attn_decode": (ctypes.c_int, [_vp] * 7 + [ctypes.c_int32] + [_vp] * 3 + [ctypes.c_int32, ctypes.c_float, AttnDims] +
                        [_vp] * 3 + [ctypes.c_size_t, _vp]),
    "moe_attn_weights": (ctypes.c_int, [_vp] * 6 + [ctypes.c_int32, _vp, ctypes.c_float, _vp, AttnDims] + [_vp] * 3),
    "moe_kv_evict": (ctypes.c_int, [_vp] * 6 + [AttnDims, ctypes.c_int32, ctypes.c_int32] + [_vp] * 7),
    "moe_kv_append_norm": (ctypes.c_int, [_vp] * 3 + [ctypes.c_int64] * 3 + [ctypes.c_int32] * 2 + [_vp, ctypes.c_int32] +
                           [_vp] * 3 + [ctypes.c_int32] * 3 + [_vp, AttnDims, _vp, _vp, ctypes.c_float] + [_vp] * 6),
    "moe_kv_append_int8": (ctypes.c_int, [_vp] * 3 + [ctypes.c_int64] * 3 + [ctypes.c_int32] * 2 + [_vp, ctypes.c_int32] +
                           [_vp] * 3 + [ctypes.c_int32] * 3 + [_vp] * 3 + [AttnDims, _vp, _vp, ctypes.c_float] + [_vp] * 6),
    "moe_kv_fork": (ctypes.c_int, [_vp] * 3 + [ctypes.c_int32, _vp, _vp, AttnDims, ctypes.c_int32, ctypes.c_int64] + [_vp] * 5),
    "moe_kv_compact": (ctypes.c_int, [_vp] * 3 + [AttnDims, ctypes.c_int32, ctypes.c_int64] + [_vp] * 5),
    "moe_stream_read_probe": (ctypes.c_int, [_vp, ctypes.c_size_t, _vp, _vp]),
    "eldr_idf": (ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp]),
    "eldr_signature": (ctypes.c_int, [_vp, _vp, ctypes.c_int32, ctypes.c_int32, _vp,
                                      ctypes.c_int32, _vp]),
    "eldr_rho": (ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int32, _vp,
                                ctypes.c_int32, _vp]),
    "eldr_greedy_layers": (ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp,
                                          _vp, ctypes.c_int32, _vp, ctypes.c_int32, _vp, _vp, _vp]),
    "eldr_balanced_kmeans": (ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                            _vp, ctypes.c_int32, _vp, _vp, _vp]),
    "eldr_route": (ctypes.c_int, [_vp, ctypes.c_int32, _vp, ctypes.c_int32, _vp, ctypes.c_float,
                                  _vp]),
    "eldr_route_batch": (ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int32,
                                        _vp, ctypes.c_float, _vp]),
}

_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library (once); raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2607_00466_amd.build`")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def header_functions(paths=HEADER_PATHS) -> list[str]:
    """Names of the functions the headers under include/ declare."""
    text = "\n".join(open(p).read() for p in paths)
    return sorted(set(re.findall(r"^\s*(?:const\s+)?\w+\*?\s+\*?((?:moe|eldr)_\w+)\s*\(", text,
                                 re.M)))


def status_string(status: int) -> str:
    return load().moe_status_string(status).decode()


def _check(fn: str, status: int) -> None:
    if status != MOE_OK:
        raise MoeError(fn, status, status_string(status))


# A decode layer of a small shape takes the GPU about 19 us, and an eager call of
# moe_layer is bound by what runs here and by its five launches.  So the checks
# below are one expression when they pass, a layer makes each of its tensors'
# checks once a call instead of once an entry point, addresses go to ctypes as
# plain integers, and the stream is looked up without a Stream object (0.4 us
# against 2.9).  Measured (tiny shape, 13 tokens, eager, on the host): 45.0 ->
# 23.1 us a layer.

def _ptr(t: torch.Tensor | None):
    return None if t is None else t.data_ptr()


# The current stream's address without a Stream object (a private name of torch's).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    """The hipStream_t of a torch stream (None: the current one)."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, numel: int) -> None:
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()
            and t.numel() >= numel):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: must be a device tensor, got {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name}: needs at least {numel} elements, has {t.numel()}")


def dims(T: int, H: int, E: int, K: int, I: int) -> MoeDims:
    return MoeDims(T, H, E, K, I)


# ----------------------------------------------------------------------------- entry points

def moe_gate_topk(x, w_gate, d: MoeDims, logits, topk_ids, topk_w, stream=None) -> None:
    _need(x, "x", torch.float32, d.T * d.H)
    _need(w_gate, "w_gate", torch.float32, d.E * d.H)
    _need(logits, "logits", torch.float32, d.T * d.E)
    _need(topk_ids, "topk_ids", torch.int32, d.T * d.K)
    _need(topk_w, "topk_w", torch.float32, d.T * d.K)
    _check("moe_gate_topk", load().moe_gate_topk(_ptr(x), _ptr(w_gate), d, _ptr(logits),
                                                 _ptr(topk_ids), _ptr(topk_w), _stream(stream)))


def moe_bucket(topk_ids, d: MoeDims, counts, offsets, perm_token, pair_pos, union_ids, union_size,
               stream=None) -> None:
    _need(topk_ids, "topk_ids", torch.int32, d.T * d.K)
    _need(counts, "counts", torch.int32, d.E)
    _need(offsets, "offsets", torch.int32, d.E + 1)
    _need(perm_token, "perm_token", torch.int32, d.T * d.K)
    _need(pair_pos, "pair_pos", torch.int32, d.T * d.K)
    _need(union_ids, "union_ids", torch.int32, 2 * d.E)
    _need(union_size, "union_size", torch.int32, 1)
    _check("moe_bucket", load().moe_bucket(_ptr(topk_ids), d, _ptr(counts), _ptr(offsets),
                                           _ptr(perm_token), _ptr(pair_pos), _ptr(union_ids),
                                           _ptr(union_size), _stream(stream)))


def moe_ffn_workspace_bytes(d: MoeDims) -> int:
    return int(load().moe_ffn_workspace_bytes(d))


def moe_expert_ffn(x, w13, w2, offsets, perm_token, union_ids, union_size, d: MoeDims, y_perm,
                   ws, stream=None) -> None:
    """The expert FFN of the union; w13 and w2 as packed by ``pack_expert_weights``."""
    _need(x, "x", torch.float32, d.T * d.H)
    _need(w13, "w13", torch.bfloat16, 2 * d.E * d.I * d.H)
    _need(w2, "w2", torch.bfloat16, d.E * d.H * d.I)
    _need(offsets, "offsets", torch.int32, d.E + 1)
    _need(perm_token, "perm_token", torch.int32, d.T * d.K)
    _need(union_ids, "union_ids", torch.int32, 2 * d.E)
    _need(union_size, "union_size", torch.int32, 1)
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn", load().moe_expert_ffn(
        _ptr(x), _ptr(w13), _ptr(w2), _ptr(offsets), _ptr(perm_token), _ptr(union_ids),
        _ptr(union_size), d, _ptr(y_perm), _ptr(ws), ws_bytes, _stream(stream)))


def _need_ws(ws, d: MoeDims) -> int:
    if ws.device.type != "cuda" or not ws.is_contiguous():
        raise ValueError("ws: must be a contiguous device tensor")
    return ws.numel() * ws.element_size()


def moe_expert_ffn_up(x, w13, offsets, perm_token, union_ids, union_size, d: MoeDims, ws,
                      stream=None) -> None:
    _need(x, "x", torch.float32, d.T * d.H)
    _need(w13, "w13", torch.bfloat16, 2 * d.E * d.I * d.H)
    _need_routing(offsets, perm_token, union_ids, union_size, d)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn_up", load().moe_expert_ffn_up(
        _ptr(x), _ptr(w13), _ptr(offsets), _ptr(perm_token), _ptr(union_ids),
        _ptr(union_size), d, _ptr(ws), ws_bytes, _stream(stream)))


def _need_buckets(d: MoeDims, counts, offsets, perm_token, pair_pos, union_ids, union_size):
    _need(counts, "counts", torch.int32, d.E)
    _need(offsets, "offsets", torch.int32, d.E + 1)
    _need(perm_token, "perm_token", torch.int32, d.T * d.K)
    _need(pair_pos, "pair_pos", torch.int32, d.T * d.K)
    _need(union_ids, "union_ids", torch.int32, 2 * d.E)
    _need(union_size, "union_size", torch.int32, 1)


def moe_expert_ffn_noalloc(x, w13, w2, offsets, perm_token, union_ids, union_size, d: MoeDims,
                           y_perm, stream=None) -> None:
    """moe_expert_ffn with the library's fixed device workspace (no caller buffer)."""
    _need(x, "x", torch.float32, d.T * d.H)
    _need(w13, "w13", torch.bfloat16, 2 * d.E * d.I * d.H)
    _need(w2, "w2", torch.bfloat16, d.E * d.H * d.I)
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    _need_routing(offsets, perm_token, union_ids, union_size, d)
    _check("moe_expert_ffn_noalloc", load().moe_expert_ffn_noalloc(
        _ptr(x), _ptr(w13), _ptr(w2), _ptr(offsets), _ptr(perm_token), _ptr(union_ids),
        _ptr(union_size), d, _ptr(y_perm), _stream(stream)))


def moe_expert_ffn_up_routed(x, w13, topk_ids, d: MoeDims, counts, offsets, perm_token, pair_pos,
                             union_ids, union_size, ws, stream=None) -> None:
    """moe_bucket then moe_expert_ffn_up, one launch for T <= 64."""
    _need(x, "x", torch.float32, d.T * d.H)
    _need(w13, "w13", torch.bfloat16, 2 * d.E * d.I * d.H)
    _need(topk_ids, "topk_ids", torch.int32, d.T * d.K)
    _need_buckets(d, counts, offsets, perm_token, pair_pos, union_ids, union_size)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn_up_routed", load().moe_expert_ffn_up_routed(
        _ptr(x), _ptr(w13), _ptr(topk_ids), d, _ptr(counts), _ptr(offsets), _ptr(perm_token),
        _ptr(pair_pos), _ptr(union_ids), _ptr(union_size), _ptr(ws), ws_bytes, _stream(stream)))


def moe_ffn_sync_bytes(d: MoeDims) -> int:
    return int(load().moe_ffn_sync_bytes(d))


def _need_sync(sync, d: MoeDims) -> None:
    _need(sync, "sync", torch.int32, moe_ffn_sync_bytes(d) // 4)


def moe_expert_ffn_routed(x, w13, w2, topk_ids, d: MoeDims, counts, offsets, perm_token, pair_pos,
                          union_ids, union_size, y_perm, ws, sync, stream=None) -> None:
    """moe_bucket then moe_expert_ffn, one launch for T <= 64.  ``sync`` is an
    int32 [64 E + 1] device tensor (moe_ffn_sync_bytes), zero before the first
    call (left zero)."""
    _need(x, "x", torch.float32, d.T * d.H)
    _need(w13, "w13", torch.bfloat16, 2 * d.E * d.I * d.H)
    _need(w2, "w2", torch.bfloat16, d.E * d.H * d.I)
    _need(topk_ids, "topk_ids", torch.int32, d.T * d.K)
    _need_buckets(d, counts, offsets, perm_token, pair_pos, union_ids, union_size)
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    ws_bytes = _need_ws(ws, d)
    _need_sync(sync, d)
    _check("moe_expert_ffn_routed", load().moe_expert_ffn_routed(
        _ptr(x), _ptr(w13), _ptr(w2), _ptr(topk_ids), d, _ptr(counts), _ptr(offsets),
        _ptr(perm_token), _ptr(pair_pos), _ptr(union_ids), _ptr(union_size), _ptr(y_perm),
        _ptr(ws), ws_bytes, _ptr(sync), _stream(stream)))


def moe_expert_ffn_down(ws, w2, offsets, perm_token, union_ids, union_size, d: MoeDims, y_perm,
                        stream=None) -> None:
    _need(w2, "w2", torch.bfloat16, d.E * d.H * d.I)
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    _need_routing(offsets, perm_token, union_ids, union_size, d)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn_down", load().moe_expert_ffn_down(
        _ptr(ws), _ptr(w2), _ptr(offsets), _ptr(perm_token), _ptr(union_ids), _ptr(union_size), d,
        ws_bytes, _ptr(y_perm), _stream(stream)))


def moe_pack_up_weights(w1, w3, dst=None, stream=None) -> torch.Tensor:
    """Pack W1 and W3 ([E, I, H] bf16 each) into one band-interleaved tensor; returns dst."""
    if w1.dim() != 3 or w1.shape != w3.shape:
        raise ValueError("w1, w3: expected two [E, I, H] tensors")
    E, I, H = (int(v) for v in w1.shape)
    _need(w1, "w1", torch.bfloat16, E * I * H)
    _need(w3, "w3", torch.bfloat16, E * I * H)
    if dst is None:
        dst = torch.empty((E, 2 * I, H), dtype=torch.bfloat16, device=w1.device)
    _need(dst, "dst", torch.bfloat16, 2 * E * I * H)
    _check("moe_pack_up_weights", load().moe_pack_up_weights(_ptr(w1), _ptr(w3), E, I, H, _ptr(dst),
                                                             _stream(stream)))
    return dst


def moe_pack_down_weights(w2, dst=None, stream=None) -> torch.Tensor:
    """Pack W2 ([E, H, I] bf16) band by band for the down projection; returns dst."""
    if w2.dim() != 3:
        raise ValueError("w2: expected [E, H, I]")
    E, H, I = (int(v) for v in w2.shape)
    _need(w2, "w2", torch.bfloat16, E * H * I)
    if dst is None:
        dst = torch.empty_like(w2)
    _need(dst, "dst", torch.bfloat16, E * H * I)
    _check("moe_pack_down_weights", load().moe_pack_down_weights(_ptr(w2), E, H, I, _ptr(dst),
                                                                 _stream(stream)))
    return dst


def pack_expert_weights(w1, w3, w2, stream=None):
    """Pack (w1 [E,I,H], w3 [E,I,H], w2 [E,H,I]) for moe_expert_ffn: returns (w13, w2p)."""
    return (moe_pack_up_weights(w1, w3, stream=stream), moe_pack_down_weights(w2, stream=stream))


# ----------------------------------------------------------------------------- MXFP4 experts
#
# An MXFP4 weight is a pair (codes, scales) of uint8 device tensors: codes
# [E, R, K/2] (two E2M1 codes a byte, the even index in the low nibble) and
# scales [E, R, K/32] (E8M0), as checkpoints store them; packed pairs are
# flat uint8 tensors of the same sizes.

def _need_u8(t, name: str, numel: int) -> None:
    _need(t, name, torch.uint8, numel)


def moe_pack_mxfp4_up(w1, w3, stream=None):
    """Pack W1 and W3 (each (codes [E,I,H/2], scales [E,I,H/32])); returns (codes, scales)."""
    (c1, s1), (c3, s3) = w1, w3
    if c1.dim() != 3:
        raise ValueError("codes: expected [E, R, K/2]")
    E, I, H = int(c1.shape[0]), int(c1.shape[1]), int(c1.shape[2]) * 2
    for name, t, n in (("w1 codes", c1, E * I * H // 2), ("w3 codes", c3, E * I * H // 2),
                       ("w1 scales", s1, E * I * H // 32), ("w3 scales", s3, E * I * H // 32)):
        _need_u8(t, name, n)
    codes = torch.empty(E * I * H, dtype=torch.uint8, device=c1.device)
    scales = torch.empty(E * I * H // 16, dtype=torch.uint8, device=c1.device)
    _check("moe_pack_mxfp4_up", load().moe_pack_mxfp4_up(
        _ptr(c1), _ptr(s1), _ptr(c3), _ptr(s3), E, I, H, _ptr(codes), _ptr(scales), _stream(stream)))
    return codes, scales


def moe_pack_mxfp4_down(w2, stream=None):
    """Pack W2 ((codes [E,H,I/2], scales [E,H,I/32])); returns (codes, scales)."""
    c2, s2 = w2
    if c2.dim() != 3:
        raise ValueError("codes: expected [E, R, K/2]")
    E, H, I = int(c2.shape[0]), int(c2.shape[1]), int(c2.shape[2]) * 2
    _need_u8(c2, "w2 codes", E * H * I // 2)
    _need_u8(s2, "w2 scales", E * H * I // 32)
    codes = torch.empty(E * H * I // 2, dtype=torch.uint8, device=c2.device)
    scales = torch.empty(E * H * I // 32, dtype=torch.uint8, device=c2.device)
    _check("moe_pack_mxfp4_down", load().moe_pack_mxfp4_down(
        _ptr(c2), _ptr(s2), E, H, I, _ptr(codes), _ptr(scales), _stream(stream)))
    return codes, scales


def pack_mxfp4_expert_weights(w1, w3, w2, stream=None):
    """Pack MXFP4 (w1, w3, w2) for moe_expert_ffn_mxfp4; returns (up, down) pairs."""
    return moe_pack_mxfp4_up(w1, w3, stream), moe_pack_mxfp4_down(w2, stream)


def _need_mx_up(up, d: MoeDims) -> None:
    _need_u8(up[0], "up codes", d.E * d.I * d.H)
    _need_u8(up[1], "up scales", d.E * d.I * d.H // 16)


def _need_mx_down(down, d: MoeDims) -> None:
    _need_u8(down[0], "down codes", d.E * d.H * d.I // 2)
    _need_u8(down[1], "down scales", d.E * d.H * d.I // 32)


def _need_routing(offsets, perm_token, union_ids, union_size, d: MoeDims) -> None:
    _need(offsets, "offsets", torch.int32, d.E + 1)
    _need(perm_token, "perm_token", torch.int32, d.T * d.K)
    _need(union_ids, "union_ids", torch.int32, 2 * d.E)
    _need(union_size, "union_size", torch.int32, 1)


def moe_expert_ffn_mxfp4(x, up, down, offsets, perm_token, union_ids, union_size, d: MoeDims,
                         y_perm, ws, stream=None) -> None:
    _need(x, "x", torch.float32, d.T * d.H)
    _need_mx_up(up, d)
    _need_mx_down(down, d)
    _need_routing(offsets, perm_token, union_ids, union_size, d)
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn_mxfp4", load().moe_expert_ffn_mxfp4(
        _ptr(x), _ptr(up[0]), _ptr(up[1]), _ptr(down[0]), _ptr(down[1]), _ptr(offsets),
        _ptr(perm_token), _ptr(union_ids), _ptr(union_size), d, _ptr(y_perm), _ptr(ws), ws_bytes,
        _stream(stream)))


def moe_expert_ffn_mxfp4_up(x, up, offsets, perm_token, union_ids, union_size, d: MoeDims, ws,
                            stream=None) -> None:
    _need(x, "x", torch.float32, d.T * d.H)
    _need_mx_up(up, d)
    _need_routing(offsets, perm_token, union_ids, union_size, d)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn_mxfp4_up", load().moe_expert_ffn_mxfp4_up(
        _ptr(x), _ptr(up[0]), _ptr(up[1]), _ptr(offsets), _ptr(perm_token), _ptr(union_ids),
        _ptr(union_size), d, _ptr(ws), ws_bytes, _stream(stream)))


def moe_expert_ffn_mxfp4_up_routed(x, up, topk_ids, d: MoeDims, counts, offsets, perm_token,
                                   pair_pos, union_ids, union_size, ws, stream=None) -> None:
    """moe_bucket then moe_expert_ffn_mxfp4_up, one launch for T <= 64."""
    _need(x, "x", torch.float32, d.T * d.H)
    _need_mx_up(up, d)
    _need(topk_ids, "topk_ids", torch.int32, d.T * d.K)
    _need_buckets(d, counts, offsets, perm_token, pair_pos, union_ids, union_size)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn_mxfp4_up_routed", load().moe_expert_ffn_mxfp4_up_routed(
        _ptr(x), _ptr(up[0]), _ptr(up[1]), _ptr(topk_ids), d, _ptr(counts), _ptr(offsets),
        _ptr(perm_token), _ptr(pair_pos), _ptr(union_ids), _ptr(union_size), _ptr(ws), ws_bytes,
        _stream(stream)))


def moe_expert_ffn_mxfp4_routed(x, up, down, topk_ids, d: MoeDims, counts, offsets, perm_token,
                                pair_pos, union_ids, union_size, y_perm, ws, sync,
                                stream=None) -> None:
    """moe_bucket then moe_expert_ffn_mxfp4, one launch for T <= 64 (``sync`` as
    for moe_expert_ffn_routed)."""
    _need(x, "x", torch.float32, d.T * d.H)
    _need_mx_up(up, d)
    _need_mx_down(down, d)
    _need(topk_ids, "topk_ids", torch.int32, d.T * d.K)
    _need_buckets(d, counts, offsets, perm_token, pair_pos, union_ids, union_size)
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    ws_bytes = _need_ws(ws, d)
    _need_sync(sync, d)
    _check("moe_expert_ffn_mxfp4_routed", load().moe_expert_ffn_mxfp4_routed(
        _ptr(x), _ptr(up[0]), _ptr(up[1]), _ptr(down[0]), _ptr(down[1]), _ptr(topk_ids), d,
        _ptr(counts), _ptr(offsets), _ptr(perm_token), _ptr(pair_pos), _ptr(union_ids),
        _ptr(union_size), _ptr(y_perm), _ptr(ws), ws_bytes, _ptr(sync), _stream(stream)))


def moe_expert_ffn_mxfp4_down(ws, down, offsets, perm_token, union_ids, union_size, d: MoeDims,
                              y_perm, stream=None) -> None:
    _need_mx_down(down, d)
    _need_routing(offsets, perm_token, union_ids, union_size, d)
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    ws_bytes = _need_ws(ws, d)
    _check("moe_expert_ffn_mxfp4_down", load().moe_expert_ffn_mxfp4_down(
        _ptr(ws), _ptr(down[0]), _ptr(down[1]), _ptr(offsets), _ptr(perm_token), _ptr(union_ids),
        _ptr(union_size), d, ws_bytes, _ptr(y_perm), _stream(stream)))


def moe_combine(y_perm, pair_pos, topk_w, d: MoeDims, out, stream=None) -> None:
    _need(y_perm, "y_perm", torch.float32, d.T * d.K * d.H)
    _need(pair_pos, "pair_pos", torch.int32, d.T * d.K)
    _need(topk_w, "topk_w", torch.float32, d.T * d.K)
    _need(out, "out", torch.float32, d.T * d.H)
    _check("moe_combine", load().moe_combine(_ptr(y_perm), _ptr(pair_pos), _ptr(topk_w), d,
                                             _ptr(out), _stream(stream)))


# ----------------------------------------------------------------------------- a whole layer

@dataclass
class LayerBuffers:
    """Device buffers of one layer invocation (allocated once, reused every step)."""

    logits: torch.Tensor
    topk_ids: torch.Tensor
    topk_w: torch.Tensor
    counts: torch.Tensor
    offsets: torch.Tensor
    perm_token: torch.Tensor
    pair_pos: torch.Tensor
    union_ids: torch.Tensor
    union_size: torch.Tensor
    y_perm: torch.Tensor
    ws: torch.Tensor
    out: torch.Tensor
    sync: torch.Tensor  # moe_expert_ffn_routed's counters: zero at allocation, left zero by every call

    @classmethod
    def allocate(cls, d: MoeDims, device="cuda") -> "LayerBuffers":
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        nbytes = moe_ffn_workspace_bytes(d)
        return cls(
            logits=torch.empty((d.T, d.E), **f32),
            topk_ids=torch.empty((d.T, d.K), **i32),
            topk_w=torch.empty((d.T, d.K), **f32),
            counts=torch.empty(d.E, **i32),
            offsets=torch.empty(d.E + 1, **i32),
            perm_token=torch.empty(max(1, d.T * d.K), **i32),
            pair_pos=torch.empty(max(1, d.T * d.K), **i32),
            union_ids=torch.empty(2 * d.E, **i32),
            union_size=torch.empty(1, **i32),
            y_perm=torch.empty((max(1, d.T * d.K), d.H), **f32),
            ws=torch.empty(max(16, nbytes) // 4, **f32),
            out=torch.empty((d.T, d.H), **f32),
            sync=torch.zeros(max(1, moe_ffn_sync_bytes(d) // 4), **i32),
        )


# How moe_layer and moe_layer_mxfp4 run the expert FFN:
#   "fused":  moe_expert_ffn_routed -- buckets, up and down projections in one launch;
#   "routed": moe_expert_ffn_up_routed (buckets + up), then moe_expert_ffn_down;
#   "split":  moe_bucket, moe_expert_ffn_up, moe_expert_ffn_down.
# All three leave the same buffers, bit for bit.
FFN_PATHS = ("fused", "routed", "split")


def _layer(ffn: str, x, w_gate, up: tuple, down: tuple, d: MoeDims, buf: LayerBuffers, routing, stream, path: str):
    """The calls of one layer, each tensor checked once: ``ffn`` is the entry
    points' prefix, ``up`` and ``down`` the weights' addresses (checked)."""
    if path not in FFN_PATHS:
        raise ValueError(f"unknown FFN path {path!r} (one of {FFN_PATHS})")
    lib, stream = load(), _stream(stream)
    T, H, E, K = d.T, d.H, d.E, d.K
    P = T * K
    f32, i32 = torch.float32, torch.int32
    _need(x, "x", f32, T * H)
    ids, w = (buf.topk_ids, buf.topk_w) if routing is None else routing
    _need(ids, "topk_ids", i32, P)
    _need(w, "topk_w", f32, P)
    _need_buckets(d, buf.counts, buf.offsets, buf.perm_token, buf.pair_pos, buf.union_ids, buf.union_size)
    _need(buf.y_perm, "y_perm", f32, P * H)
    _need(buf.out, "out", f32, T * H)
    ws_bytes = _need_ws(buf.ws, d)
    px, pids, pw, py, pws = _ptr(x), _ptr(ids), _ptr(w), _ptr(buf.y_perm), _ptr(buf.ws)
    if routing is None:
        _need(w_gate, "w_gate", f32, E * H)
        _need(buf.logits, "logits", f32, T * E)
        _check("moe_gate_topk", lib.moe_gate_topk(px, _ptr(w_gate), d, _ptr(buf.logits), pids, pw, stream))
    pair_pos = _ptr(buf.pair_pos)
    offsets, perm, union, size = _ptr(buf.offsets), _ptr(buf.perm_token), _ptr(buf.union_ids), _ptr(buf.union_size)
    buckets = (_ptr(buf.counts), offsets, perm, pair_pos, union, size)
    if path == "fused":
        _need_sync(buf.sync, d)
        fn = ffn + "_routed"
        _check(fn, getattr(lib, fn)(px, *up, *down, pids, d, *buckets, py, pws, ws_bytes, _ptr(buf.sync), stream))
    else:
        if path == "routed":
            fn = ffn + "_up_routed"
            _check(fn, getattr(lib, fn)(px, *up, pids, d, *buckets, pws, ws_bytes, stream))
        else:
            _check("moe_bucket", lib.moe_bucket(pids, d, *buckets, stream))
            fn = ffn + "_up"
            _check(fn, getattr(lib, fn)(px, *up, offsets, perm, union, size, d, pws, ws_bytes, stream))
        fn = ffn + "_down"
        _check(fn, getattr(lib, fn)(pws, *down, offsets, perm, union, size, d, ws_bytes, py, stream))
    _check("moe_combine", lib.moe_combine(py, pair_pos, pw, d, _ptr(buf.out), stream))
    return buf.out


def moe_layer(x, w_gate, w13, w2, d: MoeDims, buf: LayerBuffers, routing=None, stream=None,
              path: str = "routed"):
    """One decode-step MoE layer on one stream: gate, buckets and expert FFN
    (buckets + up projection in one launch, then down, by default: see
    FFN_PATHS), combine.

    w13 and w2 are the expert weights packed by ``pack_expert_weights``.

    ``routing=(topk_ids, topk_w)`` (int32 [T, K] and fp32 [T, K] device
    tensors) bypasses the gate: the buckets and the combine read them in place.
    Returns ``buf.out``.
    """
    _need(w13, "w13", torch.bfloat16, 2 * d.E * d.I * d.H)
    _need(w2, "w2", torch.bfloat16, d.E * d.H * d.I)
    return _layer("moe_expert_ffn", x, w_gate, (_ptr(w13),), (_ptr(w2),), d, buf, routing, stream, path)


def moe_layer_mxfp4(x, w_gate, up, down, d: MoeDims, buf: LayerBuffers, routing=None, stream=None,
                    path: str = "routed"):
    """moe_layer with MXFP4 experts: ``up`` and ``down`` from pack_mxfp4_expert_weights."""
    _need_mx_up(up, d)
    _need_mx_down(down, d)
    return _layer("moe_expert_ffn_mxfp4", x, w_gate, (_ptr(up[0]), _ptr(up[1])), (_ptr(down[0]), _ptr(down[1])), d,
                  buf, routing, stream, path)


# ----------------------------------------------------------------------------- signature cache

def moe_sig_capture(ids, token_block, layer0: int, L: int, E: int, sig, rejected=None,
                    stream=None) -> None:
    """Add one forward's picks ids [n_layers, T, K] to the int8 cache sig [num_blocks, L, E]."""
    if ids.dim() != 3:
        raise ValueError("ids: expected [n_layers, T, K]")
    n_layers, T, K = ids.shape
    if sig.dim() != 3 or tuple(sig.shape[1:]) != (L, E):
        raise ValueError("sig: expected [num_blocks, L, E]")
    _need(ids, "ids", torch.int32, n_layers * T * K)
    _need(token_block, "token_block", torch.int32, T)
    _need(sig, "sig", torch.int8, sig.numel())
    if rejected is not None:
        _need(rejected, "rejected", torch.int32, 1)
    _check("moe_sig_capture", load().moe_sig_capture(
        _ptr(ids), _ptr(token_block), n_layers, T, K, layer0, L, E, sig.shape[0], _ptr(sig),
        _ptr(rejected), _stream(stream)))


def moe_sig_reset(blocks, sig, stream=None) -> None:
    """Zero the rows of the listed blocks of sig [num_blocks, L, E]."""
    _need(blocks, "blocks", torch.int32, blocks.numel())
    _need(sig, "sig", torch.int8, sig.numel())
    nb, L, E = sig.shape
    _check("moe_sig_reset", load().moe_sig_reset(_ptr(blocks), blocks.numel(), L, E, nb, _ptr(sig),
                                                 _stream(stream)))


def moe_sig_request_counts(sig, block_table, n_blocks, out=None, stream=None) -> torch.Tensor:
    """Per-request sums of block rows: out [R, L, E] int32."""
    nb, L, E = sig.shape
    R, max_blocks = block_table.shape
    _need(sig, "sig", torch.int8, sig.numel())
    _need(block_table, "block_table", torch.int32, R * max_blocks)
    _need(n_blocks, "n_blocks", torch.int32, R)
    if out is None:
        out = torch.empty((R, L, E), dtype=torch.int32, device=sig.device)
    _need(out, "out", torch.int32, R * L * E)
    _check("moe_sig_request_counts", load().moe_sig_request_counts(
        _ptr(sig), _ptr(block_table), _ptr(n_blocks), R, max_blocks, L, E, nb, _ptr(out),
        _stream(stream)))
    return out


# ----------------------------------------------------------------------------- attention over the paged cache
#
# Caches are tensors whose first four dimensions are [num_blocks, Hkv,
# block_size, D], of torch.bfloat16, torch.float8_e4m3fn (a scale a kv head) or
# torch.int8 (a scale for each page and kv head); only the block stride may be
# larger than dense (d.block_stride), as where keys and values interleave in one
# allocation.

MOE_KV_BF16, MOE_KV_FP8, MOE_KV_INT8 = 0, 1, 3
MOE_IN_BF16, MOE_IN_FP32 = 0, 1
_KV_TYPES = {torch.bfloat16: MOE_KV_BF16, torch.float8_e4m3fn: MOE_KV_FP8, torch.int8: MOE_KV_INT8}
_KV_DTYPES = {v: k for k, v in _KV_TYPES.items()}
_IN_TYPES = {torch.bfloat16: MOE_IN_BF16, torch.float32: MOE_IN_FP32}


def _need_int32(value: int, name: str) -> None:
    """ctypes would cut a larger count to its low 32 bits."""
    if not -(1 << 31) <= value < 1 << 31:
        raise ValueError(f"{name}: {value} is no 32-bit count")


def attn_dims(R: int, Hq: int, Hkv: int, D: int, block_size: int, max_blocks: int, num_blocks: int,
              kv_dtype=torch.bfloat16, block_stride: int = 0) -> AttnDims:
    """The shape of one attention layer: R requests, Hq query heads over Hkv kv
    heads of D values, pages of block_size slots, block tables [R, max_blocks]
    into num_blocks pages of kv_dtype."""
    if kv_dtype not in _KV_TYPES:
        raise ValueError(f"kv_dtype: expected torch.bfloat16, torch.float8_e4m3fn or torch.int8, got {kv_dtype}")
    if (R | Hq | Hkv | D | block_size | max_blocks | num_blocks) >> 31 > 0:
        for name, value in zip(("R", "Hq", "Hkv", "D", "block_size", "max_blocks", "num_blocks"),
                               (R, Hq, Hkv, D, block_size, max_blocks, num_blocks)):
            _need_int32(value, name)
    return AttnDims(R, Hq, Hkv, D, block_size, max_blocks, num_blocks, _KV_TYPES[kv_dtype], block_stride)


def _need_cache(t: torch.Tensor, name: str, d: AttnDims) -> None:
    Hkv, bs, D = d.Hkv, d.block_size, d.D
    dense = Hkv * bs * D
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is _KV_DTYPES[d.kv_type]
            and t.shape == (d.num_blocks, Hkv, bs, D)
            and (t.is_contiguous() if d.block_stride in (0, dense)
                 else t.stride() == (d.block_stride, bs * D, D, 1) or t.numel() == 0)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: must be a device tensor, got {t.device}")
    if t.dtype != _KV_DTYPES[d.kv_type]:
        raise ValueError(f"{name}: expected {_KV_DTYPES[d.kv_type]}, got {t.dtype}")
    raise ValueError(f"{name}: expected {(d.num_blocks, d.Hkv, d.block_size, d.D)} with a block stride of "
                     f"{d.block_stride or dense}, got {tuple(t.shape)} with strides {t.stride()}")


def _need_opt(t, name: str, dtype: torch.dtype, numel: int) -> None:
    if t is not None:
        _need(t, name, dtype, numel)


def _need_scales(k_scale, v_scale, d: AttnDims) -> None:
    """One a kv head or none; of 8-bit integers, one for each page and kv head."""
    if d.kv_type == MOE_KV_INT8:
        if k_scale is None or v_scale is None:
            raise ValueError("k_scale and v_scale: a cache of torch.int8 has both, [num_blocks, Hkv]")
        _need(k_scale, "k_scale", torch.float32, d.num_blocks * d.Hkv)
        _need(v_scale, "v_scale", torch.float32, d.num_blocks * d.Hkv)
        return
    _need_opt(k_scale, "k_scale", torch.float32, d.Hkv)
    _need_opt(v_scale, "v_scale", torch.float32, d.Hkv)


def _stream_here(stream, t: torch.Tensor, name: str) -> int:
    """_stream, of the current device, which t has to be on: kernels run there."""
    here = torch.cuda.current_device()
    if t.get_device() != here:
        raise ValueError(f"{name}: is on {t.device}, and the current device is cuda:{here}")
    return _raw_stream(here) if stream is None and _raw_stream is not None else _stream(stream)


def _stream_of(stream, t: torch.Tensor, name: str) -> int:
    """_stream, which has to be of the device that t is on."""
    if stream is None:
        here = torch.cuda.current_device()
        if t.get_device() == here and _raw_stream is not None:
            return _raw_stream(here)
        return _stream_here(None, t, name)
    if t.device != stream.device:
        raise ValueError(f"{name}: is on {t.device}, and the stream on {stream.device}")
    return stream.cuda_stream


def _need_rows(t: torch.Tensor, name: str, T: int, heads: int, D: int) -> int:
    """A [T, heads, D] tensor whose heads and values are contiguous; its token stride."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.shape == (T, heads, D):
        token, head, value = t.stride()
        if value == 1 and head == D and T > 1:
            return token
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name}: must be a device tensor, got {t.device}")
    if t.shape != (T, heads, D):
        raise ValueError(f"{name}: expected [{T}, {heads}, {D}], got {tuple(t.shape)}")
    token, head, value = t.stride()
    if (D > 1 and value != 1) or (heads > 1 and head != D):
        raise ValueError(f"{name}: heads and values must be contiguous, got strides {t.stride()}")
    return token if T > 1 else heads * D  # one row has no stride


def _need_groups(group_start, prefix_len) -> int:
    if (group_start is None) != (prefix_len is None):
        raise ValueError("group_start and prefix_len come together")
    if group_start is None:
        return 0
    n = prefix_len.numel()
    _need(prefix_len, "prefix_len", torch.int32, n)
    _need(group_start, "group_start", torch.int32, n + 1)
    return n


def _append_rows(q, k, v, T: int, positions, pair_axis, cos, sin, d: AttnDims, q_out, interleaved: bool):
    """What the appends' calls begin with: rows, their strides and type, T, rotation."""
    Hq, Hkv, D = d.Hq, d.Hkv, d.D
    n_axes, cols = positions.shape if positions.dim() == 2 else (0, -1)
    if cols != T:
        raise ValueError(f"positions: expected [n_axes, {T}]")
    shape = cos.shape
    if len(shape) != 2 or shape != sin.shape:
        raise ValueError("cos, sin: expected two [max_pos, rot / 2] tensors")
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    max_pos, half = shape
    if pair_axis.numel() != half:
        raise ValueError(f"pair_axis: expected {half} axes, one a pair")
    dtype = k.dtype
    if dtype not in _IN_TYPES or v.dtype is not dtype or (q is not None and q.dtype is not dtype):
        raise ValueError("q, k and v: expected all torch.bfloat16 or all torch.float32")
    q_stride = pq = pq_out = 0
    if q is not None:
        q_stride = _need_rows(q, "q", T, Hq, D)
        _need(q_out, "q_out", torch.bfloat16, T * Hq * D)
        pq, pq_out = q.data_ptr(), q_out.data_ptr()
    k_stride, v_stride = _need_rows(k, "k", T, Hkv, D), _need_rows(v, "v", T, Hkv, D)
    i32, f32 = torch.int32, torch.float32
    # (their sizes are known by now: one expression where they pass)
    if not (positions.is_cuda and positions.dtype is i32 and positions.is_contiguous() and pair_axis.is_cuda and
            pair_axis.dtype is i32 and pair_axis.is_contiguous() and cos.is_cuda and cos.dtype is f32 and
            cos.is_contiguous() and sin.is_cuda and sin.dtype is f32 and sin.is_contiguous()):
        _need(positions, "positions", i32, n_axes * T)
        _need(pair_axis, "pair_axis", i32, half)
        _need(cos, "cos", f32, max_pos * half)
        _need(sin, "sin", f32, max_pos * half)
    return (pq, k.data_ptr(), v.data_ptr(), q_stride, k_stride, v_stride, _IN_TYPES[dtype], T, positions.data_ptr(), n_axes,
            pair_axis.data_ptr(), cos.data_ptr(), sin.data_ptr(), max_pos, 2 * half, 1 if interleaved else 0), pq_out


def moe_kv_append(q, k, v, positions, pair_axis, cos, sin, slots, d: AttnDims, q_out, k_cache, v_cache,
                  k_scale=None, v_scale=None, interleaved: bool = False, stream=None) -> None:
    """Rotate q [T, Hq, D] into q_out and k [T, Hkv, D] by positions [n_axes, T], and
    store k and v in the caches' slots.  q, k and v may be views of one projection's
    rows; q and q_out may be None where only keys and values are wanted."""
    T = slots.numel()
    rows, pq_out = _append_rows(q, k, v, T, positions, pair_axis, cos, sin, d, q_out, interleaved)
    _need(slots, "slots", torch.int32, T)
    _need_opt(k_scale, "k_scale", torch.float32, d.Hkv)
    _need_opt(v_scale, "v_scale", torch.float32, d.Hkv)
    _need_cache(k_cache, "k_cache", d)
    _need_cache(v_cache, "v_cache", d)
    status = load().moe_kv_append(*rows, slots.data_ptr(), d, _ptr(k_scale), _ptr(v_scale), pq_out, k_cache.data_ptr(),
                                  v_cache.data_ptr(), _stream_of(stream, k_cache, "k_cache"))
    if status:
        _check("moe_kv_append", status)


def moe_kv_append_norm(q, k, v, positions, pair_axis, cos, sin, slots, d: AttnDims, q_out, k_cache, v_cache, q_norm,
                       k_norm, eps: float = 1e-6, k_scale=None, v_scale=None, interleaved: bool = False,
                       stream=None) -> None:
    """moe_kv_append, with each head of q and k first over the root of its mean square
    and times q_norm, k_norm [D] fp32 (None: that side is not normed)."""
    T = slots.numel()
    rows, pq_out = _append_rows(q, k, v, T, positions, pair_axis, cos, sin, d, q_out, interleaved)
    _need(slots, "slots", torch.int32, T)
    _need_opt(q_norm, "q_norm", torch.float32, d.D)
    _need_opt(k_norm, "k_norm", torch.float32, d.D)
    _need_opt(k_scale, "k_scale", torch.float32, d.Hkv)
    _need_opt(v_scale, "v_scale", torch.float32, d.Hkv)
    _need_cache(k_cache, "k_cache", d)
    _need_cache(v_cache, "v_cache", d)
    status = load().moe_kv_append_norm(
        *rows, slots.data_ptr(), d, _ptr(q_norm), _ptr(k_norm), eps, _ptr(k_scale), _ptr(v_scale), pq_out, k_cache.data_ptr(),
        v_cache.data_ptr(), _stream_here(stream, k_cache, "k_cache"))
    if status:
        _check("moe_kv_append_norm", status)


def moe_kv_append_int8(q, k, v, positions, pair_axis, cos, sin, query_start, block_table, lens, d: AttnDims, q_out, k_cache,
                       v_cache, k_scale, v_scale, q_norm=None, k_norm=None, eps: float = 1e-6, interleaved: bool = False,
                       stream=None) -> None:
    """New tokens into a cache of 8-bit integers: tokens query_start[r] ..
    query_start[r + 1] - 1 go to request r's slots from lens[r] on (lens stays as it is);
    k_scale, v_scale [num_blocks, Hkv] are brought up to date.  Norms as for
    moe_kv_append_norm."""
    T = k.shape[0]
    rows, pq_out = _append_rows(q, k, v, T, positions, pair_axis, cos, sin, d, q_out, interleaved)
    _need(query_start, "query_start", torch.int32, d.R + 1)
    _need(block_table, "block_table", torch.int32, d.R * d.max_blocks)
    _need(lens, "lens", torch.int32, d.R)
    _need_opt(q_norm, "q_norm", torch.float32, d.D)
    _need_opt(k_norm, "k_norm", torch.float32, d.D)
    _need_cache(k_cache, "k_cache", d)
    _need_cache(v_cache, "v_cache", d)
    _need_scales(k_scale, v_scale, d)
    status = load().moe_kv_append_int8(
        *rows, query_start.data_ptr(), block_table.data_ptr(), lens.data_ptr(), d, _ptr(q_norm), _ptr(k_norm), eps, pq_out,
        k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), _stream_here(stream, k_cache, "k_cache"))
    if status:
        _check("moe_kv_append_int8", status)


def _need_layers(k_cache, v_cache, k_scale, v_scale, d: AttnDims):
    """The caches of one layer, or [layers, ...] of several: their count and stride."""
    layers, stride = 1, 0
    if isinstance(k_cache, torch.Tensor) and k_cache.dim() == 4:
        _need_cache(k_cache, "k_cache", d)
        _need_cache(v_cache, "v_cache", d)
    else:
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}: expected a torch tensor")
            if t.dim() != 5:
                raise ValueError(f"{name}: expected [num_blocks, Hkv, block_size, D] or [layers, ...] of it, got {tuple(t.shape)}")
            if t.shape[0] > 1 and t.stride(0) == 0 and t.numel() > 0:  # (0 would stand for dense layers)
                raise ValueError(f"{name}: an expanded tensor's layers are all the same one")
            if t.shape[0] > 0:
                _need_cache_rows(t[0], name, d)
        layers, strides = k_cache.shape[0], k_cache.stride()
        if v_cache.shape[0] != layers or v_cache.stride() != strides:
            raise ValueError("k_cache and v_cache: expected the same shape and strides")
        if layers > 1 and d.num_blocks > 0:  # (else it is of no use)
            stride = strides[0]
    if d.kv_type == MOE_KV_INT8:
        _need(k_scale, "k_scale", torch.float32, layers * d.num_blocks * d.Hkv)
        _need(v_scale, "v_scale", torch.float32, layers * d.num_blocks * d.Hkv)
    return layers, stride


def _need_cache_rows(t: torch.Tensor, name: str, d: AttnDims) -> None:
    """One layer's pages, of block stride d.block_stride (dense where that is 0)."""
    if t.is_cuda and t.dtype is _KV_DTYPES[d.kv_type] and t.shape == (d.num_blocks, d.Hkv, d.block_size, d.D):
        block = d.block_stride or d.Hkv * d.block_size * d.D
        if t.numel() == 0 or (t.stride()[1:] == (d.block_size * d.D, d.D, 1) and (t.stride(0) == block or t.shape[0] == 1)):
            return
    _need_cache(t, name, d)


def moe_kv_fork(parent, child, page, block_table, lens, d: AttnDims, k_cache, v_cache, k_scale=None, v_scale=None,
                stream=None) -> None:
    """Request child[i] becomes a copy of request parent[i] that shares its full pages;
    what the parent's last page holds is copied to page[i], in every layer of the caches
    [layers, num_blocks, Hkv, block_size, D] (or of one layer, without the first)."""
    F = parent.numel()
    i32 = torch.int32
    _need(parent, "parent", i32, F)
    _need(child, "child", i32, F)
    _need(page, "page", i32, F)
    _need(block_table, "block_table", i32, d.R * d.max_blocks)
    _need(lens, "lens", i32, d.R)
    layers, stride = _need_layers(k_cache, v_cache, k_scale, v_scale, d)
    status = load().moe_kv_fork(
        parent.data_ptr(), child.data_ptr(), page.data_ptr(), F, block_table.data_ptr(), lens.data_ptr(), d, layers, stride,
        k_cache.data_ptr(), v_cache.data_ptr(), _ptr(k_scale), _ptr(v_scale), _stream_here(stream, k_cache, "k_cache"))
    if status:
        _check("moe_kv_fork", status)


def moe_kv_compact(remap, block_table, table_out, d: AttnDims, k_cache, v_cache, k_scale=None, v_scale=None,
                   stream=None) -> None:
    """Page b moves to page remap[b] (itself: it stays; negative: it is free) in every
    layer; table_out (which may be block_table) is block_table with the pages' new
    numbers, -1 for free ones."""
    i32 = torch.int32
    _need(remap, "remap", i32, d.num_blocks)
    _need(block_table, "block_table", i32, d.R * d.max_blocks)
    _need(table_out, "table_out", i32, d.R * d.max_blocks)
    layers, stride = _need_layers(k_cache, v_cache, k_scale, v_scale, d)
    status = load().moe_kv_compact(
        remap.data_ptr(), block_table.data_ptr(), table_out.data_ptr(), d, layers, stride, k_cache.data_ptr(),
        v_cache.data_ptr(), _ptr(k_scale), _ptr(v_scale), _stream_here(stream, k_cache, "k_cache"))
    if status:
        _check("moe_kv_compact", status)


def moe_attn_workspace_bytes(d: AttnDims) -> int:
    return int(load().moe_attn_workspace_bytes(d))


def attn_workspace(d: AttnDims, device="cuda") -> torch.Tensor:
    """A workspace for moe_attn_decode (allocated once, for every layer on a stream)."""
    return torch.zeros(max(16, moe_attn_workspace_bytes(d)) // 4, dtype=torch.float32, device=device)


def moe_attn_decode(q, k_cache, v_cache, block_table, lens, d: AttnDims, out, lse, ws, group_start=None,
                    prefix_len=None, k_scale=None, v_scale=None, sinks=None, window: int = 0, scale=None,
                    stream=None) -> None:
    """Attention of one query token a request, q [R, Hq, D], over its cached tokens;
    out [R, Hq, D], lse [R, Hq] or None.  scale defaults to 1 / sqrt(D)."""
    n = d.R * d.Hq
    _need_int32(window, "window")
    _need(q, "q", torch.bfloat16, n * d.D)
    _need(out, "out", torch.bfloat16, n * d.D)
    _need_opt(lse, "lse", torch.float32, n)
    _need_cache(k_cache, "k_cache", d)
    _need_cache(v_cache, "v_cache", d)
    _need(block_table, "block_table", torch.int32, d.R * d.max_blocks)
    _need(lens, "lens", torch.int32, d.R)
    groups = _need_groups(group_start, prefix_len)
    _need_scales(k_scale, v_scale, d)
    _need_opt(sinks, "sinks", torch.float32, d.Hq)
    ws_bytes = _need_ws(ws, d)
    _check("moe_attn_decode", load().moe_attn_decode(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table), _ptr(lens), _ptr(group_start), _ptr(prefix_len),
        groups, _ptr(k_scale), _ptr(v_scale), _ptr(sinks), window, d.D ** -0.5 if scale is None else scale, d,
        _ptr(out), _ptr(lse), _ptr(ws), ws_bytes, _stream_of(stream, k_cache, "k_cache")))


def moe_attn_weights(q, k_cache, block_table, lens, lse, d: AttnDims, weights_in, weights_out, group_start=None,
                     prefix_len=None, k_scale=None, scale=None, stream=None) -> None:
    """weights_out [R, Hkv, max_blocks * block_size] = weights_in (None: zeros) plus the
    attention weight that each cached token received; lse from moe_attn_decode."""
    n, rows = d.R * d.Hq, d.R * d.Hkv * d.max_blocks * d.block_size
    _need(q, "q", torch.bfloat16, n * d.D)
    _need(lse, "lse", torch.float32, n)
    _need_cache(k_cache, "k_cache", d)
    _need(block_table, "block_table", torch.int32, d.R * d.max_blocks)
    _need(lens, "lens", torch.int32, d.R)
    groups = _need_groups(group_start, prefix_len)
    _need_opt(k_scale, "k_scale", torch.float32, d.Hkv)
    _need_opt(weights_in, "weights_in", torch.float32, rows)
    _need(weights_out, "weights_out", torch.float32, rows)
    _check("moe_attn_weights", load().moe_attn_weights(
        _ptr(q), _ptr(k_cache), _ptr(block_table), _ptr(lens), _ptr(group_start), _ptr(prefix_len), groups,
        _ptr(k_scale), d.D ** -0.5 if scale is None else scale, _ptr(lse), d, _ptr(weights_in), _ptr(weights_out),
        _stream_of(stream, k_cache, "k_cache")))


def moe_kv_evict(weights, pos, lens, seen, block_table, d: AttnDims, budget: int, recent: int, k_cache, v_cache, src,
                 new_lens, weights_out, pos_out, protect=None, stream=None) -> None:
    """Cut every request to its `budget` cached tokens of largest weight, in place
    (see include/eldr_attention.h for the order and for what moves)."""
    rows = d.R * d.Hkv * d.max_blocks * d.block_size
    _need_int32(budget, "budget")
    _need_int32(recent, "recent")
    _need(weights, "weights", torch.float32, rows)
    _need(pos, "pos", torch.int32, rows)
    _need(lens, "lens", torch.int32, d.R)
    _need(seen, "seen", torch.int32, d.R)
    _need_opt(protect, "protect", torch.int32, d.R)
    _need(block_table, "block_table", torch.int32, d.R * d.max_blocks)
    _need_cache(k_cache, "k_cache", d)
    _need_cache(v_cache, "v_cache", d)
    _need(src, "src", torch.int32, d.R * d.Hkv * budget)
    _need(new_lens, "new_lens", torch.int32, d.R)
    _need(weights_out, "weights_out", torch.float32, rows)
    _need(pos_out, "pos_out", torch.int32, rows)
    _check("moe_kv_evict", load().moe_kv_evict(
        _ptr(weights), _ptr(pos), _ptr(lens), _ptr(seen), _ptr(protect), _ptr(block_table), d, budget, recent,
        _ptr(k_cache), _ptr(v_cache), _ptr(src), _ptr(new_lens), _ptr(weights_out), _ptr(pos_out), _stream_of(stream, k_cache, "k_cache")))


# ----------------------------------------------------------------------------- calibration

def moe_stream_read_probe(buf, sink, stream=None) -> None:
    """Read all of buf once with the plain streaming kernel (measurement aid)."""
    if buf.device.type != "cuda" or not buf.is_contiguous():
        raise ValueError("buf: must be a contiguous device tensor")
    _need(sink, "sink", torch.int32, 1)
    _check("moe_stream_read_probe", load().moe_stream_read_probe(
        _ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream(stream)))


# ----------------------------------------------------------------------------- routing (host)

def _host(a, dtype):
    """A C-contiguous NumPy array of `dtype` and a pointer to it (host memory)."""
    import numpy as np

    arr = np.ascontiguousarray(a, dtype=dtype)
    return arr, ctypes.c_void_p(arr.ctypes.data)


def eldr_idf(counts):
    """IDF table [L, E] float32 from calibration counts [N, L, E]."""
    import numpy as np

    c, pc = _host(counts, np.int32)
    N, L, E = c.shape
    out = np.empty((L, E), np.float32)
    _check("eldr_idf", load().eldr_idf(pc, N, L, E, ctypes.c_void_p(out.ctypes.data)))
    return out


def eldr_signature(counts, idf, layers):
    """Signature [len(layers) * E] float32 of one request's counts [L, E]."""
    import numpy as np

    c, pc = _host(counts, np.int32)
    w, pw = _host(idf, np.float32)
    ly, pl = _host(layers, np.int32)
    L, E = c.shape
    out = np.empty(len(ly) * E, np.float32)
    _check("eldr_signature", load().eldr_signature(pc, pw, L, E, pl, len(ly),
                                                   ctypes.c_void_p(out.ctypes.data)))
    return out


def eldr_rho(S, P, pairs) -> float:
    import numpy as np

    s, ps = _host(S, np.float32)
    p, pp = _host(P, np.float32)
    pr, ppr = _host(pairs, np.int32)
    out = ctypes.c_double(0.0)
    _check("eldr_rho", load().eldr_rho(ps, s.shape[0], s.shape[1], pp, p.shape[1], ppr, pr.shape[0],
                                       ctypes.byref(out)))
    return out.value


def eldr_greedy_layers(counts, idf, P, pairs):
    """(order [L], rho curve [L], N*) of greedy layer selection."""
    import numpy as np

    c, pc = _host(counts, np.int32)
    w, pw = _host(idf, np.float32)
    p, pp = _host(P, np.float32)
    pr, ppr = _host(pairs, np.int32)
    N, L, E = c.shape
    order = np.empty(L, np.int32)
    curve = np.empty(L, np.float64)
    n_star = ctypes.c_int32(0)
    _check("eldr_greedy_layers", load().eldr_greedy_layers(
        pc, N, L, E, pw, pp, p.shape[1], ppr, pr.shape[0], ctypes.c_void_p(order.ctypes.data),
        ctypes.c_void_p(curve.ctypes.data), ctypes.byref(n_star)))
    return order, curve, n_star.value


def eldr_balanced_kmeans(S, K: int, init, max_iters: int = 50):
    """(centroids [K, d] float32, assignment [N] int32, iterations) of balanced K-means."""
    import numpy as np

    s, ps = _host(S, np.float32)
    ini, pi = _host(init, np.int32)
    N, d = s.shape
    C = np.empty((K, d), np.float32)
    assign = np.empty(N, np.int32)
    iters = ctypes.c_int32(0)
    _check("eldr_balanced_kmeans", load().eldr_balanced_kmeans(
        ps, N, d, K, pi, max_iters, ctypes.c_void_p(C.ctypes.data),
        ctypes.c_void_p(assign.ctypes.data), ctypes.byref(iters)))
    return C, assign, iters.value


def eldr_route(s, centroids, loads, tau: float) -> int:
    import numpy as np

    v, pv = _host(s, np.float32)
    c, pc = _host(centroids, np.float32)
    ld, pld = _host(loads, np.int32)
    out = ctypes.c_int32(-1)
    _check("eldr_route", load().eldr_route(pv, v.shape[0], pc, c.shape[0], pld, tau,
                                           ctypes.byref(out)))
    return out.value


def eldr_route_batch(S, centroids, loads, tau: float):
    """Route the rows of S in order; returns (workers [R], loads after routing [K])."""
    import numpy as np

    s, ps = _host(S, np.float32)
    c, pc = _host(centroids, np.float32)
    ld = np.array(loads, dtype=np.int32, copy=True)
    workers = np.empty(s.shape[0], np.int32)
    _check("eldr_route_batch", load().eldr_route_batch(
        ps, s.shape[0], s.shape[1], pc, c.shape[0], ctypes.c_void_p(ld.ctypes.data), tau,
        ctypes.c_void_p(workers.ctypes.data)))
    return workers, ld
