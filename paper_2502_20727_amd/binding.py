"""ctypes binding of the SPD C ABI (include/spd.h, include/spd_q8.h, include/spd_testing.h): same names, argument marshalling only.

Every step of the decoder-block path runs inside the HIP library; this module turns NumPy
arrays / torch tensors / Python ints into the pointers and sizes the C calls take and turns
error codes into exceptions.  PyTorch appears only as the owner of device memory and of
the stream.  If the HIP library cannot be loaded this module raises: there is no fallback.
"""
from __future__ import annotations

import array
import ctypes as C
import functools
from typing import Dict, List, Optional, Sequence

import numpy as np

from . import build
from .workloads import Workload

SPD_F32, SPD_BF16, SPD_F16, SPD_E4M3 = 0, 1, 2, 3
SPD_OK, SPD_EINVAL, SPD_EUNSUPPORTED, SPD_EHIP, SPD_ETOOBIG = 0, -1, -2, -3, -4
SPD_STATIC_WORKSPACE_BYTES = 64 << 20
SPD_ALL_RANKS = -1
SPD_Q8_MAX_K = 131071
SPD_MAX_BATCH = 64


class SpdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        detail = ""
        if code == SPD_EHIP:
            msg = lib().spd_last_hip_error()
            detail = f": {msg.decode()}" if msg else ""
        super().__init__(f"{where}: {strerror(code)} ({code}){detail}")


class spd_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "n_layers",
                                         "tp_degree", "dtype", "max_batch", "max_ctx", "max_tokens")] + \
               [("rms_eps", C.c_float), ("rope_base", C.c_float), ("act_split", C.c_int32), ("o_bias", C.c_int32)]


SPD_SPLIT_AUTO, SPD_SPLIT_ALWAYS, SPD_SPLIT_NEVER = 0, 1, 2
SPD_TIER_TP, SPD_TIER_ISB, SPD_TIER_SB, SPD_TIER_ESB = 0, 1, 2, 3


class spd_sizes(C.Structure):
    _fields_ = [("weight_bytes", C.c_size_t), ("kv_bytes", C.c_size_t), ("workspace_bytes", C.c_size_t)]


_FP = C.POINTER(C.c_float)


class spd_layer_weights(C.Structure):
    _fields_ = [(n, _FP) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")] + \
               [(n, C.c_int64) for n in ("ld_q", "ld_k", "ld_v", "ld_o", "ld_g", "ld_u", "ld_d")] + [("bo", _FP)]


class spd_taps(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "attn", "y", "u")]


class spd_pages_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "page_size", "n_pages", "dtype",
                                         "cache_dtype", "max_ctx")] + [("rope_base", C.c_float)]


class spd_pages_sizes(C.Structure):
    _fields_ = [("pool_bytes", C.c_size_t), ("rope_bytes", C.c_size_t)]


class spd_pages_plan_info(C.Structure):
    _fields_ = [("batch", C.c_int32), ("tokens", C.c_int32), ("held", C.c_int64), ("workspace_bytes", C.c_size_t)]


_lib = _torch = _int8 = _float32 = _raw_stream = _device = None
_TYPES: Dict[object, int] = {}       # SPD_* codes of torch's element types

_PROTOS = {
    "spd_create": (C.c_int, [C.POINTER(spd_config), C.POINTER(C.c_void_p)]),
    "spd_destroy": (None, [C.c_void_p]),
    "spd_get_config": (C.c_int, [C.c_void_p, C.POINTER(spd_config)]),
    "spd_get_sizes": (C.c_int, [C.c_void_p, C.POINTER(spd_sizes)]),
    "spd_last_hip_error": (C.c_char_p, []),
    "spd_strerror": (C.c_char_p, [C.c_int]),
    "spd_rank_q_heads": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
    "spd_rank_kv_heads": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
    "spd_rank_ffn_cols": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
    "spd_sync_count": (C.c_int64, [C.c_void_p, C.c_void_p]),
    "spd_mask_from_sensitivity": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_double, C.c_double, C.c_void_p,
                                            C.c_void_p]),
    "spd_pack_shard": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(spd_layer_weights), C.c_void_p]),
    "spd_pack_shard_grouped": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(spd_layer_weights), C.c_void_p, C.c_void_p,
                                         C.c_void_p]),
    "spd_pack_shard_local": (C.c_int, [C.c_void_p, C.POINTER(spd_layer_weights), C.c_void_p]),
    "spd_unpack_shard": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(spd_layer_weights)]),
    "spd_kv_pack": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]),
    "spd_kv_unpack": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]),
    "spd_workspace_init": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "spd_rank_sum": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p]),
    "spd_block_forward": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.POINTER(spd_taps)]),
    "spd_block_forward_static": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.POINTER(spd_taps)]),
    "spd_model_forward": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.POINTER(C.c_int64)]),
    "spd_model_forward_staged": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.POINTER(C.c_int64), C.c_uint32, C.c_void_p, C.c_void_p]),
    "spd_stage_timer_create": (C.c_int, [C.c_int32, C.c_int32, C.POINTER(C.c_void_p)]),
    "spd_stage_timer_read": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "spd_stage_timer_destroy": (None, [C.c_void_p]),
    "spd_mfma_probe": (C.c_int, [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "spd_read_probe": (C.c_int, [C.c_void_p, C.c_size_t, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(C.c_double)]),
    "spd_gemm_launch_size": (C.c_int, [C.c_int32]),
    "spd_gemm_panels_fit": (C.c_int, [C.c_int32]),
    "spd_act_piece_bytes": (C.c_int, [C.c_int32, C.c_int32]),
    "spd_decode_past_caches": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.c_int32]),
    "spd_down_in_tiles": (C.c_int, [C.c_void_p, C.c_int32]),
    "spd_prefill_attention_workgroups": (C.c_int, [C.c_int32]),
    "spd_decode_qkv_slices": (C.c_int, [C.c_void_p, C.c_int32]),
    "spd_gemm_tile_of": (C.c_int, [C.c_int32] * 7 + [C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
    "spd_pages_create": (C.c_int, [C.POINTER(spd_pages_config), C.POINTER(C.c_void_p)]),
    "spd_pages_destroy": (None, [C.c_void_p]),
    "spd_pages_get_sizes": (C.c_int, [C.c_void_p, C.POINTER(spd_pages_sizes)]),
    "spd_pages_rope_table": (C.c_int, [C.c_void_p, C.c_void_p]),
    "spd_pages_plan": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                 C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)]),
    "spd_pages_plan_get_info": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(spd_pages_plan_info)]),
    "spd_pages_write": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_int64, C.c_void_p]),
    "spd_pages_read": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "spd_pages_attention": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64,
                                      C.c_void_p, C.c_void_p]),
    "spd_q8_norm": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_float,
                              C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "spd_q8_rows": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "spd_q8_swiglu": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "spd_q8_weight_bytes": (C.c_size_t, [C.c_int32, C.c_int32]),
    "spd_q8_pack": (C.c_int, [C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]),
    "spd_q8_pack_codes": (C.c_int, [C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "spd_q8_unpack": (C.c_int, [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "spd_q8_matmul_workspace": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32]),
    "spd_q8_kernel_of": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int64]),
    "spd_q8_matmul": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
}
EXPORTS = tuple(_PROTOS)
STAGES = {"prep": 0, "qkv": 1, "attn": 2, "o": 3, "gateup": 4, "down": 5}
SPD_ALL_STAGES = (1 << len(STAGES)) - 1
SPD_STAGE_EMPTY = len(STAGES)


def lib():
    """The loaded HIP library.  Raises if it is missing and cannot be built."""
    global _lib, _torch, _int8, _float32, _raw_stream, _device
    if _lib is None:
        path = build.ensure_hip()
        # PyTorch ships its own HIP runtime.  The library must bind to the same one as the tensors it
        # is handed, so torch (when installed) is imported before the library is loaded: loaded the
        # other way round, the process holds two runtimes and this library's calls see no device.
        try:
            import torch
            _torch, _int8, _float32 = torch, torch.int8, torch.float32
            _raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
            _TYPES.update({torch.float32: SPD_F32, torch.bfloat16: SPD_BF16, torch.float16: SPD_F16})
        except ImportError:
            pass
        l = C.CDLL(path)
        for name, (res, args) in _PROTOS.items():
            fn = getattr(l, name)          # AttributeError if the symbol is not exported
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


def strerror(code: int) -> str:
    return lib().spd_strerror(code).decode()


def _check(code: int, where: str) -> None:
    if code != SPD_OK:
        raise SpdError(code, where)


def _ptr(x) -> Optional[int]:
    """Address of a torch tensor / NumPy array / raw int; None stays NULL."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        assert x.flags.c_contiguous
        return x.ctypes.data
    assert x.is_contiguous()
    return x.data_ptr()


def _i32(values: Sequence[int]):
    arr = (C.c_int32 * max(len(values), 1))(*[int(v) for v in values])
    return arr


# --------------------------------------------------------------------------- host-only calls

def make_config(w: Workload, max_batch: Optional[int] = None, max_ctx: Optional[int] = None,
                max_tokens: Optional[int] = None, act_split: int = 0, o_bias: int = 0) -> spd_config:
    mb = max_batch if max_batch is not None else w.batch
    mc = max_ctx if max_ctx is not None else (w.ctx + 31) // 32 * 32
    mt = max_tokens if max_tokens is not None else max(w.batch * w.q_len, mb)
    return spd_config(w.hidden, w.n_q_heads, w.n_kv_heads, w.head_dim, w.ffn, w.n_layers, w.tp, w.dtype,
                      mb, mc, mt, w.rms_eps, w.rope_base, act_split, o_bias)


def spd_create(cfg: spd_config) -> int:
    out = C.c_void_p()
    _check(lib().spd_create(C.byref(cfg), C.byref(out)), "spd_create")
    return out.value


def spd_destroy(ctx: int) -> None:
    lib().spd_destroy(ctx)


def spd_get_sizes(ctx: int) -> spd_sizes:
    s = spd_sizes()
    _check(lib().spd_get_sizes(ctx, C.byref(s)), "spd_get_sizes")
    return s


def spd_get_config(ctx: int) -> spd_config:
    c = spd_config()
    _check(lib().spd_get_config(ctx, C.byref(c)), "spd_get_config")
    return c


def _range_call(fn, ctx, rank):
    a, b = C.c_int32(), C.c_int32()
    _check(fn(ctx, rank, C.byref(a), C.byref(b)), fn.__name__)
    return a.value, b.value


def spd_rank_q_heads(ctx: int, rank: int):
    return _range_call(lib().spd_rank_q_heads, ctx, rank)


def spd_rank_kv_heads(ctx: int, rank: int):
    return _range_call(lib().spd_rank_kv_heads, ctx, rank)


def spd_rank_ffn_cols(ctx: int, rank: int):
    return _range_call(lib().spd_rank_ffn_cols, ctx, rank)


def spd_sync_count(ctx: int, mask: Sequence[int]) -> int:
    m = np.ascontiguousarray(mask, dtype=np.uint8)
    n = lib().spd_sync_count(ctx, m.ctypes.data)
    if n < 0:
        raise SpdError(int(n), "spd_sync_count")
    return int(n)


def spd_mask_from_sensitivity(sensitivity: Sequence[float], n_spd: int, tau1: float, tau2: float):
    """Returns (mask, tier), two lists of n_layers ints."""
    s = np.ascontiguousarray(sensitivity, dtype=np.float64)
    mask = np.zeros(s.size, dtype=np.uint8)
    tier = np.zeros(s.size, dtype=np.uint8)
    _check(lib().spd_mask_from_sensitivity(s.ctypes.data if s.size else None, s.size, int(n_spd), float(tau1),
                                           float(tau2), mask.ctypes.data, tier.ctypes.data),
           "spd_mask_from_sensitivity")
    return mask.tolist(), tier.tolist()


def _weights_struct(W: Dict[str, np.ndarray]) -> spd_layer_weights:
    s = spd_layer_weights()
    for name in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2"):
        a = W[name]
        assert a.dtype == np.float32 and a.flags.c_contiguous, name
        setattr(s, name, a.ctypes.data_as(_FP))
    for name, ld in (("wq", "ld_q"), ("wk", "ld_k"), ("wv", "ld_v"), ("wo", "ld_o"), ("wg", "ld_g"),
                     ("wu", "ld_u"), ("wd", "ld_d")):
        setattr(s, ld, W[name].shape[1])
    if W.get("bo") is not None:          # bias of the output projection (block with bias)
        assert W["bo"].dtype == np.float32 and W["bo"].flags.c_contiguous
        s.bo = W["bo"].ctypes.data_as(_FP)
    return s


def spd_pack_shard(ctx: int, rank: int, dense: Dict[str, np.ndarray], out: Optional[np.ndarray] = None) -> np.ndarray:
    if out is None:
        out = np.empty(spd_get_sizes(ctx).weight_bytes, dtype=np.uint8)
    s = _weights_struct(dense)
    _check(lib().spd_pack_shard(ctx, rank, C.byref(s), out.ctypes.data), "spd_pack_shard")
    return out


def spd_pack_shard_grouped(ctx: int, rank: int, dense: Dict[str, np.ndarray], kv_heads: Optional[Sequence[int]],
                           mlp_of_rank: Optional[Sequence[int]], out: Optional[np.ndarray] = None) -> np.ndarray:
    if out is None:
        out = np.empty(spd_get_sizes(ctx).weight_bytes, dtype=np.uint8)
    s = _weights_struct(dense)
    kh = None if kv_heads is None else np.ascontiguousarray(kv_heads, dtype=np.int32)
    mr = None if mlp_of_rank is None else np.ascontiguousarray(mlp_of_rank, dtype=np.int32)
    _check(lib().spd_pack_shard_grouped(ctx, rank, C.byref(s), None if kh is None else kh.ctypes.data,
                                        None if mr is None else mr.ctypes.data, out.ctypes.data), "spd_pack_shard_grouped")
    return out


def spd_pack_shard_local(ctx: int, shard: Dict[str, np.ndarray], out: Optional[np.ndarray] = None) -> np.ndarray:
    if out is None:
        out = np.empty(spd_get_sizes(ctx).weight_bytes, dtype=np.uint8)
    s = _weights_struct(shard)
    _check(lib().spd_pack_shard_local(ctx, C.byref(s), _ptr(out)), "spd_pack_shard_local")
    return out


def spd_unpack_shard(ctx: int, packed: np.ndarray, shapes: Dict[str, tuple]) -> Dict[str, np.ndarray]:
    out = {k: np.zeros(v, dtype=np.float32) for k, v in shapes.items()}
    s = _weights_struct(out)
    _check(lib().spd_unpack_shard(ctx, packed.ctypes.data, C.byref(s)), "spd_unpack_shard")
    return out


def spd_kv_pack(ctx: int, k: np.ndarray, v: np.ndarray, cache_host: np.ndarray) -> None:
    assert k.dtype == np.float32 and v.dtype == np.float32 and k.shape == v.shape
    batch, _, n_pos, _ = k.shape
    k, v = np.ascontiguousarray(k), np.ascontiguousarray(v)      # (held until the call is over)
    _check(lib().spd_kv_pack(ctx, _ptr(k), _ptr(v), batch, n_pos, cache_host.ctypes.data), "spd_kv_pack")


def spd_kv_unpack(ctx: int, cache_host: np.ndarray, batch: int, n_pos: int, kv_heads: int, head_dim: int):
    k = np.zeros((batch, kv_heads, n_pos, head_dim), dtype=np.float32)
    v = np.zeros_like(k)
    _check(lib().spd_kv_unpack(ctx, cache_host.ctypes.data, batch, n_pos, k.ctypes.data, v.ctypes.data), "spd_kv_unpack")
    return k, v


# --------------------------------------------------------------------------- device calls

def _current_stream() -> int:
    """torch's current stream on its current device, without the object around it (which takes as long as a small launch)."""
    if _raw_stream is None or _device is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def spd_workspace_init(ctx: int, workspace, stream=None) -> None:
    _check(lib().spd_workspace_init(ctx, _ptr(workspace), _stream_ptr(stream)), "spd_workspace_init")


def spd_rank_sum(ctx: int, base, slots, n_slots: int, n_elems: int, out, stream=None) -> None:
    _check(lib().spd_rank_sum(ctx, _ptr(base), _ptr(slots), n_slots, n_elems, _ptr(out), _stream_ptr(stream)),
           "spd_rank_sum")


def spd_block_forward(ctx: int, layer: int, spd_flag: int, rank: int, packed_weights, kv_cache,
                      positions: Sequence[int], batch: int, q_len: int, x_in, slots, x_out, workspace,
                      stream=None, taps: Optional[Dict[str, object]] = None) -> None:
    t = None
    if taps:
        t = spd_taps(*[_ptr(taps.get(n)) for n in ("q", "attn", "y", "u")])
    _check(lib().spd_block_forward(ctx, layer, spd_flag, rank, _ptr(packed_weights), _ptr(kv_cache),
                                   C.cast(_i32(positions), C.c_void_p), batch, q_len, _ptr(x_in), _ptr(slots),
                                   _ptr(x_out), _ptr(workspace), _stream_ptr(stream),
                                   C.byref(t) if t is not None else None), "spd_block_forward")


def spd_block_forward_static(ctx: int, layer: int, spd_flag: int, rank: int, packed_weights, kv_cache,
                             positions: Sequence[int], batch: int, q_len: int, x_in, slots, x_out,
                             stream=None, taps: Optional[Dict[str, object]] = None) -> None:
    t = None
    if taps:
        t = spd_taps(*[_ptr(taps.get(n)) for n in ("q", "attn", "y", "u")])
    _check(lib().spd_block_forward_static(ctx, layer, spd_flag, rank, _ptr(packed_weights), _ptr(kv_cache),
                                          C.cast(_i32(positions), C.c_void_p), batch, q_len, _ptr(x_in), _ptr(slots),
                                          _ptr(x_out), _stream_ptr(stream), C.byref(t) if t is not None else None),
           "spd_block_forward_static")


def spd_model_forward(ctx: int, spd_mask: Sequence[int], rank: int, layer_weights: Sequence, layer_kv: Sequence,
                      positions: Sequence[int], batch: int, q_len: int, x_in, slots, x_out, workspace,
                      stream=None) -> int:
    mask = np.ascontiguousarray(spd_mask, dtype=np.uint8)
    n = len(layer_weights)
    wp = (C.c_void_p * n)(*[_ptr(t) for t in layer_weights])
    kp = (C.c_void_p * n)(*[_ptr(t) for t in layer_kv])
    syncs = C.c_int64(0)
    _check(lib().spd_model_forward(ctx, mask.ctypes.data, rank, C.cast(wp, C.c_void_p), C.cast(kp, C.c_void_p),
                                   C.cast(_i32(positions), C.c_void_p), batch, q_len, _ptr(x_in), _ptr(slots),
                                   _ptr(x_out), _ptr(workspace), _stream_ptr(stream), C.byref(syncs)),
           "spd_model_forward")
    return syncs.value


def spd_model_forward_staged(ctx: int, spd_mask: Sequence[int], rank: int, layer_weights: Sequence, layer_kv: Sequence,
                             positions: Sequence[int], batch: int, q_len: int, x_in, slots, x_out, workspace,
                             stage_mask: int = SPD_ALL_STAGES, timer: Optional[int] = None, stream=None,
                             layer_out=None) -> int:
    mask = np.ascontiguousarray(spd_mask, dtype=np.uint8)
    n = len(layer_weights)
    wp = (C.c_void_p * n)(*[_ptr(t) for t in layer_weights])
    kp = (C.c_void_p * n)(*[_ptr(t) for t in layer_kv])
    syncs = C.c_int64(0)
    _check(lib().spd_model_forward_staged(ctx, mask.ctypes.data, rank, C.cast(wp, C.c_void_p), C.cast(kp, C.c_void_p),
                                          C.cast(_i32(positions), C.c_void_p), batch, q_len, _ptr(x_in), _ptr(slots),
                                          _ptr(x_out), _ptr(workspace), _stream_ptr(stream), C.byref(syncs),
                                          int(stage_mask), timer, _ptr(layer_out)),
           "spd_model_forward_staged")
    return syncs.value


def spd_stage_timer_create(stage: int, max_records: int) -> int:
    out = C.c_void_p()
    _check(lib().spd_stage_timer_create(stage, max_records, C.byref(out)), "spd_stage_timer_create")
    return out.value


def spd_stage_timer_read(timer: int):
    """(launches timed, mean microseconds, min microseconds) since the last read."""
    n, mean, mn = C.c_int32(), C.c_double(), C.c_double()
    _check(lib().spd_stage_timer_read(timer, C.byref(n), C.byref(mean), C.byref(mn)), "spd_stage_timer_read")
    return n.value, mean.value, mn.value


def spd_stage_timer_destroy(timer: int) -> None:
    lib().spd_stage_timer_destroy(timer)


SPD_MFMA_PROBE_SCRATCH_BYTES = 256 * 512 * 4 + 16


def spd_mfma_probe(iters: int, random_data: bool, scratch, stream=None):
    """(TFLOP/s, shader MHz) of register-resident 16x16x32 fp16 MFMAs over a full grid; `scratch` is a device
    tensor of at least SPD_MFMA_PROBE_SCRATCH_BYTES."""
    assert scratch.is_cuda and scratch.numel() * scratch.element_size() >= SPD_MFMA_PROBE_SCRATCH_BYTES
    tf, mhz = C.c_double(), C.c_double()
    _check(lib().spd_mfma_probe(iters, 1 if random_data else 0, scratch.data_ptr(), _stream_ptr(stream), C.byref(tf),
                                C.byref(mhz)), "spd_mfma_probe")
    return tf.value, mhz.value


def spd_read_probe(buf, chunk_bytes: int, n_chunks: int, reps: int, sink, stream=None) -> float:
    """Mean microseconds per launch of a kernel that only reads chunk_bytes (device tensors `buf`, `sink`)."""
    assert buf.is_cuda and buf.numel() * buf.element_size() >= chunk_bytes * n_chunks and sink.is_cuda
    us = C.c_double()
    _check(lib().spd_read_probe(buf.data_ptr(), chunk_bytes, n_chunks, reps, sink.data_ptr(), _stream_ptr(stream), C.byref(us)),
           "spd_read_probe")
    return us.value


def spd_gemm_launch_size(n_tiles: int) -> int:
    """Workgroups launched for `n_tiles` tiles of the GEMM's tile order."""
    n = lib().spd_gemm_launch_size(n_tiles)
    if n < 0:
        _check(n, "spd_gemm_launch_size")
    return n


def spd_gemm_tile_of(TN: int, TM: int, rn: int, rm: int, tile0: int, n_tiles: int, b: int):
    """(tn, tm) of the tile that workgroup `b` takes, or None for a spare workgroup."""
    tn, tm = C.c_int32(), C.c_int32()
    rc = lib().spd_gemm_tile_of(TN, TM, rn, rm, tile0, n_tiles, b, C.byref(tn), C.byref(tm))
    if rc == 1:
        return None
    _check(rc, "spd_gemm_tile_of")
    return tn.value, tm.value


# --------------------------------------------------------------------------- 8-bit serving operators (spd_q8.h)

def spd_pages_create(cfg: spd_pages_config) -> int:
    out = C.c_void_p()
    _check(lib().spd_pages_create(C.byref(cfg), C.byref(out)), "spd_pages_create")
    return out.value


def spd_pages_destroy(pages: int) -> None:
    lib().spd_pages_destroy(pages)


def spd_pages_get_sizes(pages: int) -> spd_pages_sizes:
    s = spd_pages_sizes()
    _check(lib().spd_pages_get_sizes(pages, C.byref(s)), "spd_pages_get_sizes")
    return s


def spd_pages_rope_table(pages: int) -> np.ndarray:
    """The rotary table, fp32, flat: [max_ctx][head_dim / 2][cos, sin]."""
    out = np.empty(spd_pages_get_sizes(pages).rope_bytes // 4, dtype=np.float32)
    _check(lib().spd_pages_rope_table(pages, out.ctypes.data), "spd_pages_rope_table")
    return out


def _int32(x, what: str) -> np.ndarray:
    """Whole numbers as a contiguous int32 array."""
    if isinstance(x, (list, tuple)):          # (checks every number, faster than NumPy takes them up)
        return np.frombuffer(array.array("i", x), dtype=np.int32)
    a = np.asarray(x)
    if a.dtype != np.int32 and a.size:
        if a.dtype.kind not in "iu":
            raise TypeError(f"{what}: whole numbers wanted, not {a.dtype}")
        if int(a.min()) < -(1 << 31) or int(a.max()) >= 1 << 31:
            raise ValueError(f"{what}: beyond 32 bits")
    return np.ascontiguousarray(a, dtype=np.int32)


def spd_pages_plan(pages: int, positions: Sequence[int], q_lens: Sequence[int], page_table, window: int = 0,
                   sinks: int = 0) -> np.ndarray:
    """The plan of a step (bytes on the host).  page_table: int32 [batch, entries], or a list of lists of pages."""
    pos, lens = _int32(positions, "positions"), _int32(q_lens, "q_lens")
    if pos.shape != lens.shape or pos.ndim != 1:
        raise ValueError("positions and q_lens are lists of one length")
    if isinstance(page_table, np.ndarray):
        table = _int32(page_table, "page_table")
    else:
        # (the rest of a shorter list is of no page: a sequence that needs it is refused)
        rows = [_int32(r, "page_table") for r in page_table]
        table = np.full((len(rows), max(map(len, rows), default=0)), -1, dtype=np.int32)
        for b, r in enumerate(rows):
            table[b, :len(r)] = r
    if table.ndim != 2 or table.shape[0] != len(pos):
        raise ValueError("page_table has a row for each sequence")
    if table.size == 0:                       # (an address that is not NULL)
        table = np.full((len(pos), 1), -1, dtype=np.int32)
    for what, n in (("window", window), ("sinks", sinks)):
        if not -(1 << 31) <= n < 1 << 31:     # (ctypes would drop what does not fit)
            raise ValueError(f"{what}: beyond 32 bits")
    need = C.c_size_t(0)

    def call(out, n):
        _check(lib().spd_pages_plan(pages, len(pos), pos.ctypes.data, lens.ctypes.data, table.ctypes.data, table.shape[1], int(window),
                                    int(sinks), out, n, C.byref(need)), "spd_pages_plan")
    call(None, 0)
    plan = np.empty(need.value, dtype=np.uint8)
    call(plan.ctypes.data, plan.size)
    return plan


def spd_pages_plan_get_info(pages: int, plan: np.ndarray) -> spd_pages_plan_info:
    i = spd_pages_plan_info()
    _check(lib().spd_pages_plan_get_info(pages, plan.ctypes.data, C.byref(i)), "spd_pages_plan_get_info")
    return i


def _type(t) -> int:
    """SPD_* code of a torch tensor's element type."""
    code = _TYPES.get(t.dtype)
    if code is None:
        if _lib is None:
            lib()                # fills the table
            return _type(t)
        raise TypeError(f"float32, bfloat16 or float16 elements wanted, not {t.dtype}")
    return code


def _rows(t, shape, what: str):
    """(address, row stride) of a device matrix whose rows are contiguous; (None, 0) for None."""
    if t is None:
        return None, 0
    if t.shape != shape:
        raise ValueError(f"{what}: {shape} wanted, not {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{what}: a tensor on the device wanted")
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{what}: rows have to be contiguous, strides {t.stride()}")
    if ld < shape[1] and shape[0] == 1:
        ld = shape[1]
    return t.data_ptr(), ld


def _buffer(t, what: str = "buffer", nbytes: int = 0):
    """Address of a contiguous device tensor of at least `nbytes`, None for None."""
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{what}: a contiguous tensor on the device wanted")
    if t.nbytes < nbytes:
        raise ValueError(f"{what}: too small")
    return t.data_ptr()


def _like(t, other, what: str):
    if t is not None and t.dtype is not other.dtype:
        raise TypeError(f"{what}: {other.dtype} wanted, not {t.dtype}")


def spd_pages_write(pages: int, plan: "PagePlan", qkv, rope, pool, q_out=None, stream=None) -> None:
    """qkv [tokens, (q_heads + 2 kv_heads) head_dim]; q_out [tokens, q_heads head_dim] in the pool's 16-bit type, or None."""
    width = qkv.shape[-1]
    p, ld = _rows(qkv, (plan.tokens, width), "qkv")
    if width < plan.qkv_cols:
        raise ValueError("qkv: rows too short")
    qo, ld_q = _rows(q_out, plan.q_shape, "q_out")
    if qo is not None and _type(q_out) != plan.dtype:
        raise TypeError("q_out: the pool's 16-bit type wanted")
    rc = _lib.spd_pages_write(pages, plan.host_ptr, plan.device_ptr, _type(qkv), p, ld, _buffer(rope, "rope", plan.rope_bytes),
                              _buffer(pool, "pool", plan.pool_bytes), qo, ld_q,
                              _current_stream() if stream is None else _stream_ptr(stream))
    if rc:
        raise SpdError(rc, "spd_pages_write")


def spd_pages_read(pages: int, plan: "PagePlan", pool, k_out, v_out, stream=None) -> None:
    """k_out, v_out [held, kv_heads, head_dim]: every position of every sequence, one after the other."""
    if k_out.shape != plan.held_shape or v_out.shape != plan.held_shape:
        raise ValueError(f"k_out, v_out: {plan.held_shape} wanted")
    _like(v_out, k_out, "v_out")
    rc = _lib.spd_pages_read(pages, plan.host_ptr, plan.device_ptr, _buffer(pool, "pool", plan.pool_bytes), _type(k_out),
                             _buffer(k_out, "k_out"), _buffer(v_out, "v_out"),
                             _current_stream() if stream is None else _stream_ptr(stream))
    if rc:
        raise SpdError(rc, "spd_pages_read")


def spd_pages_attention(pages: int, plan: "PagePlan", q, pool, out, workspace=None, stream=None) -> None:
    """q, out [tokens, q_heads head_dim] in the pool's 16-bit type, rows may be strided."""
    qp, ld_q = _rows(q, plan.q_shape, "q")
    op, ld_o = _rows(out, plan.q_shape, "out")
    if _type(q) != plan.dtype or _type(out) != plan.dtype:
        raise TypeError("q, out: the pool's 16-bit type wanted")
    rc = _lib.spd_pages_attention(pages, plan.host_ptr, plan.device_ptr, qp, ld_q, _buffer(pool, "pool", plan.pool_bytes), op, ld_o,
                                  _buffer(workspace, "workspace", plan.workspace_bytes),
                                  _current_stream() if stream is None else _stream_ptr(stream))
    if rc:
        raise SpdError(rc, "spd_pages_attention")


def _codes(codes, scales, shape):
    if codes.dtype is not _int8 or scales.dtype is not _float32 or scales.numel() != shape[0] or not (scales.is_cuda and scales.is_contiguous()):
        raise TypeError("codes: int8, scales: contiguous float32 on the device, one a row")
    return _rows(codes, shape, "codes")


def spd_q8_norm(x, add, gain, eps: float, sum_out, codes, scales, stream=None) -> None:
    """codes, scales <- RMSNorm(x + add) * gain in 8 bits; sum_out <- x + add.  add and sum_out may be None."""
    l = _lib or lib()
    rows, n = shape = x.shape
    px, lx = _rows(x, shape, "x")
    pa, la = _rows(add, shape, "add")
    ps, ls = _rows(sum_out, shape, "sum_out")
    pc, lc = _codes(codes, scales, shape)
    _like(add, x, "add")
    _like(sum_out, x, "sum_out")
    if gain.dtype is not _float32 or gain.numel() != n:
        raise TypeError("gain: float32, one a column")
    rc = l.spd_q8_norm(_type(x), rows, n, px, lx, pa, la, _buffer(gain, "gain"), eps, ps, ls, pc, lc, scales.data_ptr(),
                       _current_stream() if stream is None else _stream_ptr(stream))
    if rc:
        raise SpdError(rc, "spd_q8_norm")


def spd_q8_rows(x, codes, scales, stream=None) -> None:
    l = _lib or lib()
    rows, n = shape = x.shape
    px, lx = _rows(x, shape, "x")
    pc, lc = _codes(codes, scales, shape)
    rc = l.spd_q8_rows(_type(x), rows, n, px, lx, pc, lc, scales.data_ptr(), _current_stream() if stream is None else _stream_ptr(stream))
    if rc:
        raise SpdError(rc, "spd_q8_rows")


def spd_q8_swiglu(x, codes, scales, stream=None) -> None:
    """x [rows, 2 n]: gates, then ups."""
    l = _lib or lib()
    rows, n = x.shape
    n //= 2
    px, lx = _rows(x, (rows, 2 * n), "x")
    pc, lc = _codes(codes, scales, (rows, n))
    rc = l.spd_q8_swiglu(_type(x), rows, n, px, lx, pc, lc, scales.data_ptr(), _current_stream() if stream is None else _stream_ptr(stream))
    if rc:
        raise SpdError(rc, "spd_q8_swiglu")


@functools.lru_cache(maxsize=None)
def spd_q8_weight_bytes(K: int, N: int) -> int:
    return lib().spd_q8_weight_bytes(K, N)


def _packed_host(a: np.ndarray, K: int, N: int) -> np.ndarray:
    if not a.flags.c_contiguous or a.nbytes < spd_q8_weight_bytes(K, N):
        raise ValueError("packed weights: a contiguous array of spd_q8_weight_bytes(K, N) bytes wanted")
    return a


def spd_q8_pack(w: np.ndarray, out: Optional[np.ndarray] = None) -> np.ndarray:
    """Quantises and packs fp32 weights [K, N] (y = x W)."""
    assert w.dtype == np.float32 and w.ndim == 2 and w.flags.c_contiguous
    K, N = w.shape
    if out is None:
        out = np.empty(spd_q8_weight_bytes(K, N), dtype=np.uint8)
    _check(lib().spd_q8_pack(K, N, w.ctypes.data, N, _packed_host(out, K, N).ctypes.data), "spd_q8_pack")
    return out


def spd_q8_pack_codes(w: np.ndarray, w_scale: np.ndarray, out: Optional[np.ndarray] = None) -> np.ndarray:
    assert w.dtype == np.int8 and w.ndim == 2 and w.flags.c_contiguous and w_scale.dtype == np.float32 and w_scale.shape == w.shape[1:]
    K, N = w.shape
    if out is None:
        out = np.empty(spd_q8_weight_bytes(K, N), dtype=np.uint8)
    scale = np.ascontiguousarray(w_scale)     # (held until the call is over)
    _check(lib().spd_q8_pack_codes(K, N, w.ctypes.data, N, scale.ctypes.data, _packed_host(out, K, N).ctypes.data), "spd_q8_pack_codes")
    return out


def spd_q8_unpack(K: int, N: int, packed: np.ndarray):
    """(codes int8 [K, N], scales fp32 [N]) of packed weights."""
    w, s = np.empty((K, N), dtype=np.int8), np.empty(N, dtype=np.float32)
    _check(lib().spd_q8_unpack(K, N, _packed_host(packed, K, N).ctypes.data, w.ctypes.data, N, s.ctypes.data), "spd_q8_unpack")
    return w, s


@functools.lru_cache(maxsize=4096)
def spd_q8_matmul_workspace(rows: int, K: int, N: int) -> int:
    return lib().spd_q8_matmul_workspace(rows, K, N)


def spd_q8_kernel_of(rows: int, K: int, N: int, ld_codes: Optional[int] = None) -> int:
    rc = lib().spd_q8_kernel_of(rows, K, N, (K + 15) // 16 * 16 if ld_codes is None else ld_codes)
    if rc < 0:
        raise SpdError(rc, "spd_q8_kernel_of")
    return rc


def spd_q8_matmul(codes, scales, packed, N: int, add, out, workspace=None, stream=None) -> None:
    """out [rows, N] <- (codes [rows, K] times the packed K x N weights) * scales (+ add)."""
    l = _lib or lib()
    rows, K = codes.shape
    shape = (rows, N)
    pc, lc = _codes(codes, scales, (rows, K))
    pa, la = _rows(add, shape, "add")
    po, lo = _rows(out, shape, "out")
    _like(add, out, "add")
    rc = l.spd_q8_matmul(rows, K, N, pc, lc, scales.data_ptr(), _buffer(packed, "packed", spd_q8_weight_bytes(K, N)), _type(out), pa, la, po, lo,
                         _buffer(workspace, "workspace"),
                         _current_stream() if stream is None else _stream_ptr(stream))
    if rc:
        raise SpdError(rc, "spd_q8_matmul")


# --------------------------------------------------------------------------- device-memory plumbing

class DeviceShard:
    """Device buffers (torch tensors) of one rank, or of all ranks back to back, for a workload.

    Holds memory only; every computation goes through the spd_* calls above.
    """

    def __init__(self, w: Workload, ranks: Sequence[int], device, max_ctx: Optional[int] = None,
                 max_tokens: Optional[int] = None, max_batch: Optional[int] = None, act_split: int = 0,
                 o_bias: int = 0):
        import torch
        self.torch = torch
        self.w = w
        self.ranks = list(ranks)
        self.device = device
        self.cfg = make_config(w, max_batch=max_batch, max_ctx=max_ctx, max_tokens=max_tokens, act_split=act_split,
                               o_bias=o_bias)
        self.ctx = spd_create(self.cfg)
        self.sizes = spd_get_sizes(self.ctx)
        nr = len(self.ranks)
        u8 = torch.uint8
        self.weights = [torch.empty(nr * self.sizes.weight_bytes, dtype=u8, device=device) for _ in range(w.n_layers)]
        self.kv = [torch.zeros(nr * self.sizes.kv_bytes, dtype=u8, device=device) for _ in range(w.n_layers)]
        self.workspace = torch.zeros(self.sizes.workspace_bytes, dtype=u8, device=device)
        spd_workspace_init(self.ctx, self.workspace)

    def close(self):
        if self.ctx:
            spd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def load_layer(self, layer: int, shards: List[Dict[str, np.ndarray]]) -> None:
        """Pack (host) and upload the given ranks' shards of one layer."""
        torch = self.torch
        wb = self.sizes.weight_bytes
        host = np.empty(len(shards) * wb, dtype=np.uint8)
        for i, s in enumerate(shards):
            spd_pack_shard_local(self.ctx, s, host[i * wb:(i + 1) * wb])
        self.weights[layer].copy_(torch.from_numpy(host))

    def load_kv(self, layer: int, kvs: List[tuple]) -> None:
        """kvs[i] = (k, v) natural-layout prefill of rank i: [batch, kv, n_pos, d] fp32."""
        torch = self.torch
        kb = self.sizes.kv_bytes
        host = np.zeros(len(kvs) * kb, dtype=np.uint8)
        for i, (k, v) in enumerate(kvs):
            spd_kv_pack(self.ctx, k, v, host[i * kb:(i + 1) * kb])
        self.kv[layer].copy_(torch.from_numpy(host))

    def read_kv(self, layer: int, rank_index: int, batch: int, n_pos: int):
        kb = self.sizes.kv_bytes
        host = self.kv[layer][rank_index * kb:(rank_index + 1) * kb].cpu().numpy()
        return spd_kv_unpack(self.ctx, host, batch, n_pos, self.w.kv_per_rank, self.w.head_dim)

    def rank_arg(self) -> int:
        return SPD_ALL_RANKS if len(self.ranks) > 1 else self.ranks[0]


class DevicePages:
    """A pool of pages on the device with its handle and rotary table.  Holds memory only; a pool made here is cleared on torch's current
    stream, which other streams wait for."""

    def __init__(self, cfg: spd_pages_config, device, pool=None, rope: bool = True):
        import torch
        self.cfg = cfg
        self.ctx = None
        self.ctx = spd_pages_create(cfg)
        self.sizes = spd_pages_get_sizes(self.ctx)
        self.device = device
        if pool is not None and pool.numel() * pool.element_size() < self.sizes.pool_bytes:
            raise ValueError("pool: too small for the configuration")
        self.pool = pool if pool is not None else torch.zeros(self.sizes.pool_bytes, dtype=torch.uint8, device=device)
        self.rope = torch.from_numpy(spd_pages_rope_table(self.ctx)).to(device) if rope else None

    def close(self):
        if self.ctx:
            spd_pages_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PagePlan:
    """The plan of a step, on the host and on the device, and its scratch, cleared on torch's current stream.  Calls of one plan that may
    overlap (on several streams) need a scratch each; the object has to live until its calls are over.

    Every step needs one (35 to 85 us on the host).  The copy to the device waits for what torch's current stream was given before: plan a step
    ahead of the launches of the one before it where the device is to stay busy."""

    def __init__(self, pages: DevicePages, positions: Sequence[int], q_lens: Sequence[int], page_table, window: int = 0, sinks: int = 0):
        import torch
        self.pages = pages
        self.host = spd_pages_plan(pages.ctx, positions, q_lens, page_table, window, sinks)
        self.info = spd_pages_plan_get_info(pages.ctx, self.host)
        self.device = torch.from_numpy(self.host).to(pages.device)
        c = pages.cfg
        self.tokens, self.workspace_bytes, self.dtype = self.info.tokens, self.info.workspace_bytes, c.dtype
        self.qkv_cols = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim
        self.q_shape, self.held_shape = (self.tokens, c.n_q_heads * c.head_dim), (self.info.held, c.n_kv_heads, c.head_dim)
        self.pool_bytes, self.rope_bytes = pages.sizes.pool_bytes, pages.sizes.rope_bytes
        self.host_ptr, self.device_ptr = self.host.ctypes.data, self.device.data_ptr()
        n = self.workspace_bytes
        self.workspace = torch.zeros(n, dtype=torch.uint8, device=pages.device) if n else None
