"""Thin Python binding of the NetKV C ABI (``include/netkv.h``).

Argument marshalling only: every function forwards to the entry point of the
same name in ``libnetkv.so``; all computation happens in the CUDA kernels
behind it.  Device buffers may be given as torch tensors (their ``data_ptr()``
is passed) or as raw integer device addresses; ``None`` passes NULL.  A
non-OK status raises :class:`NetKVError`.  There is no CPU fallback: if the
library is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnetkv.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it first "
                      "(python -c 'import __graft_entry__ as g; g.build()')")
_lib = C.CDLL(LIB_PATH)

NETKV_OK, NETKV_EINVAL, NETKV_ENOMEM, NETKV_ECUDA, NETKV_ELIMIT = 0, 1, 2, 3, 4
NETKV_PREFIX_MATCH_STATIC_MAX_R = 524288
NETKV_DEV_EDOMAIN, NETKV_DEV_EFULL, NETKV_DEV_ERANGE = 1, 2, 4
NETKV_DEV_ETIMEOUT = 8
_NAMES = {1: "NETKV_EINVAL", 2: "NETKV_ENOMEM", 3: "NETKV_ECUDA",
          4: "NETKV_ELIMIT (more requests than the fixed scratch of netkv_prefix_match_static holds)"}

EXPORTS = ("netkv_topology_create", "netkv_topology_destroy", "netkv_topology_query",
           "netkv_oracle_build", "netkv_oracle_build_directed", "netkv_oracle_build_tiers",
           "netkv_cache_index_bytes",
           "netkv_cache_build",
           "netkv_prefix_match_workspace_size",
           "netkv_prefix_match", "netkv_prefix_match_static", "netkv_schedule_workspace_size",
           "netkv_schedule_streams", "netkv_schedule_streams_util",
           "netkv_schedule_streams_inflight",
           "netkv_schedule_inflight_workspace_size",
           "netkv_schedule_streams_load",
           "netkv_lru_state_bytes", "netkv_lru_init", "netkv_lru_export",
           "netkv_schedule_streams_evolving",
           "netkv_copy_async", "netkv_copy_group_async",
           "netkv_kv_store", "netkv_kv_load", "netkv_attn_prompt",
           "netkv_attn_decode_workspace_size", "netkv_attn_decode", "netkv_kv_evict",
           "netkv_version")


class NetKVError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} returned {_NAMES.get(code, code)}")
        self.code = code


class _Desc(C.Structure):
    _fields_ = [("fanout", C.c_uint32 * 4), ("role", C.c_void_p),
                ("tier_bw_Bps", C.c_double * 4), ("tier_lat_s", C.c_double * 4),
                ("n_links", C.c_uint32)]


# netkv_weights, 32 bytes: 4 x f32, i64, u64
WEIGHTS_DTYPE = np.dtype([("w_net", "<f4"), ("w_prefix", "<f4"), ("w_load", "<f4"),
                          ("theta_s_per_token", "<f4"), ("cap_tokens", "<i8"),
                          ("bytes_per_token", "<u8")])
assert WEIGHTS_DTYPE.itemsize == 32

_P, _U32, _U64, _F64 = C.c_void_p, C.c_uint32, C.c_uint64, C.c_double
_lib.netkv_version.restype = C.c_uint32
_lib.netkv_topology_create.argtypes = [C.POINTER(_Desc), C.POINTER(C.c_void_p)]
_lib.netkv_topology_destroy.argtypes = [_P]
_lib.netkv_topology_query.argtypes = [_P, _P, _P, _P, _P]
_lib.netkv_oracle_build.argtypes = [_P, _P, _U32, _F64, _P, _P, _P, _P]
_lib.netkv_oracle_build_directed.argtypes = [_P, _P, _P, _U32, _F64, _P, _P, _P, _P]
_lib.netkv_oracle_build_tiers.argtypes = [_P, _P, _U32, _F64, _P, _P, _P, _P]
_lib.netkv_cache_index_bytes.argtypes = [_U32, _U32, _U32]
_lib.netkv_cache_index_bytes.restype = C.c_size_t
_lib.netkv_cache_build.argtypes = [_P, _U32, _U32, _U32, _P, _P, _P, _P]
_lib.netkv_prefix_match_workspace_size.argtypes = [_U32]
_lib.netkv_prefix_match_workspace_size.restype = C.c_size_t
_lib.netkv_prefix_match.argtypes = [_P, _U32, _U32, _U32, _P, _P, _U32, _P, _P, C.c_size_t, _P,
                                    _P, _P]
_lib.netkv_prefix_match_static.argtypes = [_P, _U32, _U32, _U32, _P, _P, _U32, _P, _P, _P, _P]
_lib.netkv_schedule_workspace_size.argtypes = [_U32, _U32]
_lib.netkv_schedule_workspace_size.restype = C.c_size_t
_lib.netkv_schedule_streams.argtypes = [_P, _U32, _P, _U32, _P, _P, _P, _P, _P, _U32, _P, _P,
                                        _P, _P, _P, _P, _P, _P, C.c_size_t, _P, _P]
_lib.netkv_schedule_streams_util.argtypes = [_P, _U32, _P, _U32, _P, _P, _P, _P, _P, _U32, _P,
                                             _P, _P, _P, _P, _P, _P, _P, C.c_size_t, _P, _P]
_lib.netkv_schedule_streams_inflight.argtypes = [_P, _U32, _P, _U32, _P, _P, _P, _P, _P, _P,
                                                 _U32, _P, _P, _U32, _P, _P, _P, _P, _P, _P,
                                                 _P, C.c_size_t, _P, _P]
_lib.netkv_schedule_inflight_workspace_size.argtypes = [_U32, _U32]
_lib.netkv_schedule_inflight_workspace_size.restype = C.c_size_t
class LoadModel(C.Structure):
    """netkv_load_model: the paper's compute-load model constants (Sec. III-C, IV-B)."""
    _fields_ = [("t_a_s", C.c_float), ("t_b_s", C.c_float), ("beta_max", C.c_int32),
                ("reserved", C.c_int32), ("m_min_bytes", C.c_int64), ("m0_bytes", C.c_int64)]


_lib.netkv_schedule_streams_load.argtypes = [_P, _U32, _P, C.POINTER(LoadModel), _U32, _P, _P,
                                             _P, _P, _P, _U32, _P, _P, _P, _P, _P, _P, _P, _P,
                                             _P, _P, _P]
class LruConfig(C.Structure):
    """netkv_lru_config: capacity and table sizes of the evolving (LRU) decode caches."""
    _fields_ = [("cap_blocks", C.c_uint64), ("log2_slots", C.c_uint32), ("log2_ring", C.c_uint32)]


def lru_config(cap_blocks: int) -> LruConfig:
    """The smallest tables netkv.h allows for caches of cap_blocks blocks."""
    need = int(cap_blocks) + 65536
    ls = 4
    while (3 << ls) // 4 < need - 1:
        ls += 1
    lr = 4
    while (1 << lr) < need:
        lr += 1
    return LruConfig(int(cap_blocks), ls, lr)


_lib.netkv_lru_state_bytes.argtypes = [_U64, C.POINTER(LruConfig)]
_lib.netkv_lru_state_bytes.restype = C.c_size_t
_lib.netkv_lru_init.argtypes = [_P, C.c_size_t, _U64, C.POINTER(LruConfig), _P, _P, _P, _P]
_lib.netkv_lru_export.argtypes = [_P, C.c_size_t, _U64, C.POINTER(LruConfig), _P, _P, _P, _P]
_lib.netkv_schedule_streams_evolving.argtypes = [_P, _U32, _P, _U32, _P, _P, _P, _P, _U32, _P, _P,
                                                 _P, _P, _P, C.c_size_t, C.POINTER(LruConfig), _P,
                                                 _P, _P, _P, _P, _P, _P, _P]
_lib.netkv_copy_async.argtypes = [_P, _P, C.c_size_t, _P]
_lib.netkv_copy_group_async.argtypes = [_P, _U32, _P]
NETKV_BLOCK_TOKENS = 16
NETKV_F16, NETKV_BF16 = 0, 1
NETKV_KV_INT8, NETKV_KV_E4M3 = 0, 1
_KV_FORMATS = {"int8": NETKV_KV_INT8, "float8_e4m3fn": NETKV_KV_E4M3}
_lib.netkv_kv_store.argtypes = [_P, _U32, _P, _U64, _P, _U64, _U32, _P, _U64, _P, _P, _U32, _P, _P]
_lib.netkv_kv_load.argtypes = _lib.netkv_kv_store.argtypes
_lib.netkv_attn_prompt.argtypes = [_U32, _P, _U64, _P, _U64, _P, _U64, _U32, _U32, _U32, _U32, _P,
                                   _P, _U64, _U64, C.c_float, _P, _U64, _P, _P, _P]
_lib.netkv_attn_decode_workspace_size.argtypes = [_P, _U32, _U32, _U32, C.c_int]
_lib.netkv_attn_decode_workspace_size.restype = C.c_size_t
_lib.netkv_attn_decode.argtypes = [_P, _U32, _P, _U64, _U32, _U32, _P, _P, _U32, C.c_float, _P,
                                   _U64, _P, _P, _P, _P, C.c_size_t, _P, _P]
_lib.netkv_kv_evict.argtypes = [_U32, _P, _P, _P, _U32, _P, _U32, _U32, _P, _P, _P, _P, _P, _P, _P]
for _f in EXPORTS:
    if _f not in ("netkv_version", "netkv_prefix_match_workspace_size", "netkv_cache_index_bytes",
                  "netkv_schedule_workspace_size", "netkv_schedule_inflight_workspace_size",
                  "netkv_lru_state_bytes", "netkv_attn_decode_workspace_size"):
        getattr(_lib, _f).restype = C.c_int


class KvPages(C.Structure):
    """netkv_kv_pages over four tensors, which it keeps: codes [n_pages, kv_heads, 16, dim] of
    torch.int8 or torch.float8_e4m3fn, and fp32 scales [n_pages, kv_heads]."""
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_k_scale", C.c_void_p),
                ("d_v_scale", C.c_void_p), ("n_pages", C.c_uint32), ("kv_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("format", C.c_uint32)]

    def __init__(self, k, v, k_scale, v_scale):
        fmt = str(k.dtype).replace("torch.", "")
        if fmt not in _KV_FORMATS or v.dtype != k.dtype:
            raise TypeError(f"KV pages of {k.dtype} and {v.dtype}: int8 or float8_e4m3fn expected")
        if k.dim() != 4 or k.shape[2] != NETKV_BLOCK_TOKENS or v.shape != k.shape:
            raise ValueError("KV pages are [n_pages, kv_heads, 16, dim]")
        if k_scale.shape != k.shape[:2] or v_scale.shape != k.shape[:2]:
            raise ValueError("KV scales are [n_pages, kv_heads]")
        for t in (k, v, k_scale, v_scale):
            if not t.is_contiguous():
                raise ValueError("KV pages and scales are contiguous")
            if t.get_device() != k.get_device():
                raise ValueError("KV pages and scales of one device expected")
        if not _ROWS:
            _ask_torch()
        for t in (k_scale, v_scale):
            if t.dtype not in _F32:
                raise TypeError(f"float32 tensor expected, got {t.dtype}")
        super().__init__(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                         k.shape[0], k.shape[1], k.shape[3], _KV_FORMATS[fmt])
        self.tensors = (k, v, k_scale, v_scale)
        self.ref = C.byref(self)
        self.heads_dim = (k.shape[1], k.shape[3])  # a field of a structure takes longer to read
        self.device, self.device_index = k.device, k.get_device()


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return int(x.data_ptr())


_torch = None


def current_stream() -> Optional[int]:
    """torch's current CUDA stream, or None before CUDA is initialised."""
    global _torch
    if _torch is None:
        import torch as _torch  # once: an import statement takes 0.3 us a call
    torch = _torch
    if not torch.cuda.is_initialized():
        return None
    # the raw handle, without a Stream object around it (1.6 -> 0.4 us a call)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _stream(s) -> Optional[int]:
    if s is None:
        return current_stream()
    if isinstance(s, int):
        return s
    return int(s.cuda_stream)


def _check(fn: str, code: int) -> None:
    if code != NETKV_OK:
        raise NetKVError(fn, code)


def netkv_version() -> int:
    return int(_lib.netkv_version())


class Topology:
    """Owns a netkv_topology_t handle (released by netkv_topology_destroy)."""

    def __init__(self, handle: int):
        self.handle = handle

    @property
    def as_parameter(self):
        return self.handle

    def __del__(self):
        if getattr(self, "handle", None):
            try:
                _lib.netkv_topology_destroy(self.handle)
            except Exception:
                pass
            self.handle = None


def netkv_topology_create(fanout: Sequence[int], role: np.ndarray, tier_bw_Bps: Sequence[float],
                          tier_lat_s: Sequence[float], n_links: int) -> Topology:
    role = np.ascontiguousarray(role, dtype=np.uint8)
    d = _Desc()
    d.fanout[:] = [int(x) for x in fanout]
    d.role = role.ctypes.data
    d.tier_bw_Bps[:] = [float(x) for x in tier_bw_Bps]
    d.tier_lat_s[:] = [float(x) for x in tier_lat_s]
    d.n_links = int(n_links)
    h = C.c_void_p()
    _check("netkv_topology_create", _lib.netkv_topology_create(C.byref(d), C.byref(h)))
    return Topology(h.value)


def netkv_topology_destroy(topo: Topology) -> None:
    if topo.handle:
        _check("netkv_topology_destroy", _lib.netkv_topology_destroy(topo.handle))
        topo.handle = None


def netkv_topology_query(topo: Topology):
    v = [C.c_uint32() for _ in range(4)]
    _check("netkv_topology_query",
           _lib.netkv_topology_query(topo.handle, *[C.byref(x) for x in v]))
    return tuple(int(x.value) for x in v)


def netkv_oracle_build(topo: Topology, util, n_snap: int, kv_bytes: float, C_out=None, UB=None,
                       status=None, stream=None) -> None:
    _check("netkv_oracle_build", _lib.netkv_oracle_build(
        topo.handle, _ptr(util), int(n_snap), float(kv_bytes), _ptr(C_out), _ptr(UB),
        _ptr(status), _stream(stream)))


def netkv_cache_index_bytes(n_sets: int, D: int, log2_capacity: int) -> int:
    return int(_lib.netkv_cache_index_bytes(int(n_sets), int(D), int(log2_capacity)))


def netkv_cache_build(index, n_sets: int, D: int, log2_capacity: int, keys, key_off, status=None,
                      stream=None) -> None:
    _check("netkv_cache_build", _lib.netkv_cache_build(
        _ptr(index), int(n_sets), int(D), int(log2_capacity), _ptr(keys), _ptr(key_off),
        _ptr(status), _stream(stream)))


def netkv_prefix_match_workspace_size(R: int) -> int:
    return int(_lib.netkv_prefix_match_workspace_size(int(R)))


def netkv_prefix_match(index, D: int, log2_capacity: int, n_sets: int, chains, chain_off, R: int,
                       set_off, M, status=None, stream=None, workspace=None) -> None:
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check("netkv_prefix_match", _lib.netkv_prefix_match(
        _ptr(index), int(D), int(log2_capacity), int(n_sets), _ptr(chains), _ptr(chain_off),
        int(R), _ptr(set_off), _ptr(workspace), ws_bytes, _ptr(M), _ptr(status), _stream(stream)))


def netkv_prefix_match_static(index, D: int, log2_capacity: int, n_sets: int, chains, chain_off,
                              R: int, set_off, M, status=None, stream=None) -> None:
    """Prefix match that allocates nothing (fixed device scratch inside the library);
    for callers that may not allocate device memory.  Overlapping calls race."""
    _check("netkv_prefix_match_static", _lib.netkv_prefix_match_static(
        _ptr(index), int(D), int(log2_capacity), int(n_sets), _ptr(chains), _ptr(chain_off),
        int(R), _ptr(set_off), _ptr(M), _ptr(status), _stream(stream)))


def netkv_schedule_workspace_size(R: int, D: int) -> int:
    return int(_lib.netkv_schedule_workspace_size(int(R), int(D)))


def netkv_schedule_streams(topo: Topology, n_streams: int, weights, R: int, length, prefill, snap,
                           M, UB, n_snap: int, events, event_off, load_init, dec, best, second,
                           load_final, status=None, stream=None, workspace=None) -> None:
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check("netkv_schedule_streams", _lib.netkv_schedule_streams(
        topo.handle, int(n_streams), _ptr(weights), int(R), _ptr(length), _ptr(prefill),
        _ptr(snap), _ptr(M), _ptr(UB), int(n_snap), _ptr(events), _ptr(event_off),
        _ptr(load_init), _ptr(dec), _ptr(best), _ptr(second), _ptr(load_final), _ptr(workspace),
        ws_bytes, _ptr(status), _stream(stream)))


def netkv_schedule_streams_util(topo: Topology, n_streams: int, weights, R: int, length, prefill,
                                snap, M, util, n_snap: int, events, event_off, load_init, dec,
                                best, second, load_final, status=None, stream=None,
                                workspace=None) -> None:
    """The greedy with level bottlenecks from the utilisation rows; see include/netkv.h."""
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check("netkv_schedule_streams_util", _lib.netkv_schedule_streams_util(
        topo.handle, int(n_streams), _ptr(weights), int(R), _ptr(length), _ptr(prefill),
        _ptr(snap), _ptr(M), _ptr(util), int(n_snap), _ptr(events), _ptr(event_off),
        _ptr(load_init), _ptr(dec), _ptr(best), _ptr(second), _ptr(load_final), _ptr(workspace),
        ws_bytes, _ptr(status), _stream(stream)))


def netkv_schedule_streams_inflight(topo: Topology, n_streams: int, weights, R: int, length,
                                    prefill, snap, arrival_us, M, UB, n_snap: int, events,
                                    event_off, inflight_cap: int, load_init, dec, best, second,
                                    xfer_us, load_final, status=None, stream=None,
                                    workspace=None) -> None:
    """Algorithm 1 with self-contention; see include/netkv.h."""
    ws_bytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check("netkv_schedule_streams_inflight", _lib.netkv_schedule_streams_inflight(
        topo.handle, int(n_streams), _ptr(weights), int(R), _ptr(length), _ptr(prefill),
        _ptr(snap), _ptr(arrival_us), _ptr(M), _ptr(UB), int(n_snap), _ptr(events),
        _ptr(event_off), int(inflight_cap), _ptr(load_init), _ptr(dec), _ptr(best),
        _ptr(second), _ptr(xfer_us), _ptr(load_final), _ptr(workspace), ws_bytes, _ptr(status),
        _stream(stream)))


def netkv_schedule_inflight_workspace_size(R: int, D: int) -> int:
    return int(_lib.netkv_schedule_inflight_workspace_size(int(R), int(D)))


def netkv_oracle_build_directed(topo: Topology, util_up, util_down, n_snap: int, kv_bytes: float,
                                C=None, UB=None, status=None, stream=None) -> None:
    """Oracle build with directed links; see include/netkv.h."""
    _check("netkv_oracle_build_directed", _lib.netkv_oracle_build_directed(
        topo.handle, _ptr(util_up), _ptr(util_down), int(n_snap), float(kv_bytes), _ptr(C),
        _ptr(UB), _ptr(status), _stream(stream)))


def netkv_oracle_build_tiers(topo: Topology, c, n_snap: int, kv_bytes: float, C=None, UB=None,
                             status=None, stream=None) -> None:
    """The paper-literal per-tier oracle; see include/netkv.h."""
    _check("netkv_oracle_build_tiers", _lib.netkv_oracle_build_tiers(
        topo.handle, _ptr(c), int(n_snap), float(kv_bytes), _ptr(C), _ptr(UB), _ptr(status),
        _stream(stream)))


def netkv_schedule_streams_load(topo: Topology, n_streams: int, weights, model: LoadModel, R: int,
                                length, prefill, snap, M, UB, n_snap: int, events, event_off,
                                m_init, n_init, dec, best, second, m_final, n_final,
                                status=None, stream=None) -> None:
    """Algorithm 1 with the paper's compute-load model; see include/netkv.h."""
    _check("netkv_schedule_streams_load", _lib.netkv_schedule_streams_load(
        topo.handle, int(n_streams), _ptr(weights), C.byref(model), int(R), _ptr(length),
        _ptr(prefill), _ptr(snap), _ptr(M), _ptr(UB), int(n_snap), _ptr(events), _ptr(event_off),
        _ptr(m_init), _ptr(n_init), _ptr(dec), _ptr(best), _ptr(second), _ptr(m_final),
        _ptr(n_final), _ptr(status), _stream(stream)))


def netkv_lru_state_bytes(n_caches: int, cfg: LruConfig) -> int:
    return int(_lib.netkv_lru_state_bytes(int(n_caches), C.byref(cfg)))


def _nbytes(t) -> int:
    return int(t.numel() * t.element_size())


def netkv_lru_init(state, n_caches: int, cfg: LruConfig, keys, key_off, status=None,
                   stream=None) -> None:
    """Evolving caches from key lists (most recently used first); see include/netkv.h."""
    _check("netkv_lru_init", _lib.netkv_lru_init(_ptr(state), _nbytes(state), int(n_caches),
                                                 C.byref(cfg), _ptr(keys), _ptr(key_off),
                                                 _ptr(status), _stream(stream)))


def netkv_lru_export(state, n_caches: int, cfg: LruConfig, keys_out, len_out, status=None,
                     stream=None) -> None:
    """Every evolving cache's blocks, most recently used first; see include/netkv.h."""
    _check("netkv_lru_export", _lib.netkv_lru_export(_ptr(state), _nbytes(state), int(n_caches),
                                                     C.byref(cfg), _ptr(keys_out), _ptr(len_out),
                                                     _ptr(status), _stream(stream)))


def netkv_schedule_streams_evolving(topo: Topology, n_streams: int, weights, R: int, length,
                                    prefill, snap, UB, n_snap: int, chains, chain_off, events,
                                    event_off, state, cfg: LruConfig, load_init, dec, best,
                                    second, M, load_final, status=None, stream=None) -> None:
    """Algorithm 1 with evolving LRU caches; see include/netkv.h."""
    _check("netkv_schedule_streams_evolving", _lib.netkv_schedule_streams_evolving(
        topo.handle, int(n_streams), _ptr(weights), int(R), _ptr(length), _ptr(prefill),
        _ptr(snap), _ptr(UB), int(n_snap), _ptr(chains), _ptr(chain_off), _ptr(events),
        _ptr(event_off), _ptr(state), _nbytes(state), C.byref(cfg), _ptr(load_init), _ptr(dec),
        _ptr(best),
        _ptr(second), _ptr(M), _ptr(load_final), _ptr(status), _stream(stream)))


def netkv_copy_async(dst, src, nbytes: int, stream=None) -> None:
    """Kernel copy between device and/or pinned host buffers (torch tensors or addresses)."""
    _check("netkv_copy_async", _lib.netkv_copy_async(_ptr(dst), _ptr(src), int(nbytes),
                                                     _stream(stream)))


def netkv_copy_group_async(copies, stream=None) -> None:
    """Kernel copies (dst, src, bytes), each as for netkv_copy_async, in one launch per 32."""
    flat = [v for dst, src, nbytes in copies for v in (_ptr(dst) or 0, _ptr(src) or 0, int(nbytes))]
    _check("netkv_copy_group_async", _lib.netkv_copy_group_async(
        (_U64 * len(flat))(*flat), len(flat) // 3, _stream(stream)))


# ---- KV blocks: tensors carry their sizes, so these take them from the tensors and check that
# they fit together and are all on the current CUDA device, on which the kernels run; everything else
# is checked behind the entry points.

# What is asked of torch, once (a program without it may use the rest of the binding): the dtypes
# of each kind, and who knows the current device and its stream.
_ROWS, _F32, _I32, _I64 = {}, (), (), ()
_raw_stream = _current_device = None


def _ask_torch() -> None:
    global _F32, _I32, _I64, _raw_stream, _current_device
    import torch
    _ROWS.update({torch.float16: NETKV_F16, torch.bfloat16: NETKV_BF16})
    _F32, _I32, _I64 = (torch.float32,), (torch.int32, torch.uint32), (torch.int64, torch.uint64)
    _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _device(t) -> int:
    """The device of a call's first tensor, which has to be the current one: its kernels run there.
    The other tensors are compared with it one by one."""
    if not _ROWS:
        _ask_torch()
    d = t.get_device()
    if d < 0:
        raise TypeError(f"CUDA tensors expected, got one on {t.device}")
    if d != _current_device():
        raise ValueError(f"tensors on CUDA device {d}, but the current one is {_current_device()}")
    return d


def _elsewhere(t, device: int) -> None:
    raise ValueError(f"tensors on CUDA device {device} expected, got one on {t.device}")


def _rows(t, heads: int, dim: int, device: int, code: Optional[int] = None):
    """(dtype code, address, row stride) of rows [rows, heads, dim]; a row is contiguous."""
    c = _ROWS.get(t.dtype)
    if c is None:
        raise TypeError(f"float16 or bfloat16 rows expected, got {t.dtype}")
    if code is not None and c != code:
        raise TypeError("tensors of one dtype expected")
    n, h, d = t.shape
    if h != heads or d != dim:
        raise ValueError(f"rows of {(heads, dim)} expected, got {(h, d)}")
    if t.get_device() != device:
        _elsewhere(t, device)
    if t.is_contiguous():
        return c, t.data_ptr(), h * d
    s, sh, sd = t.stride()
    if (sd != 1 and d > 1) or (sh != d and h > 1):
        raise ValueError("a row's heads have to lie one after another")
    return c, t.data_ptr(), s if n > 1 else h * d


def _ints(t, kind: tuple, n: int, device: int) -> Optional[int]:
    """The address of a contiguous integer tensor of n entries."""
    if t is None:
        return None
    if t.dtype not in kind:
        raise TypeError(f"{32 if kind is _I32 else 64}-bit integers expected, got {t.dtype}")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"a contiguous tensor of {n} entries expected, got {tuple(t.shape)}")
    if t.get_device() != device:
        _elsewhere(t, device)
    return t.data_ptr()


def _table(t, n_seqs: int, device: int):
    shape = t.shape
    if len(shape) != 2 or shape[0] != n_seqs:
        raise ValueError(f"a block table of {n_seqs} rows expected, got {tuple(shape)}")
    width = shape[1]
    return _ints(t, _I32, n_seqs * width, device), width


def _plane(t, rows: int, width: int, device: int) -> Optional[int]:
    """The address of a contiguous fp32 tensor of that shape."""
    if t is None:
        return None
    if t.dtype not in _F32:
        raise TypeError(f"float32 tensor expected, got {t.dtype}")
    if t.shape != (rows, width) or not t.is_contiguous():
        raise ValueError(f"a contiguous tensor of {(rows, width)} expected, got {tuple(t.shape)}")
    if t.get_device() != device:
        _elsewhere(t, device)
    return t.data_ptr()


def _word(t, device: int) -> Optional[int]:
    """The address of a status word: a tensor (in pinned host memory too, where a program may read it
    without a copy), an address, or None."""
    if t is None or t.__class__ is int:
        return t
    if t.get_device() != device and not t.is_pinned():
        _elsewhere(t, device)
    return t.data_ptr()


def _on_stream(device: int, stream) -> Optional[int]:
    """The given stream, else torch's current one on the device."""
    return _raw_stream(device) if stream is None else _stream(stream)


def _kv_move(fn: str, call, pages: KvPages, k, v, off, start, table, status, stream) -> None:
    heads, dim = pages.heads_dim
    d = _device(k)
    if pages.device_index != d:
        _elsewhere(pages, d)
    dt, kp, ks = _rows(k, heads, dim, d)
    _, vp, vs = _rows(v, heads, dim, d, dt)
    rows = k.shape[0]
    if v.shape[0] != rows:
        raise ValueError("as many rows of keys as of values expected")
    n = off.numel() - 1
    tp, tw = _table(table, n, d)
    code = call(pages.ref, dt, kp, ks, vp, vs, n, _ints(off, _I64, n + 1, d), rows,
                _ints(start, _I32, n, d), tp, tw, _word(status, d), _on_stream(d, stream))
    if code:
        raise NetKVError(fn, code)


def netkv_kv_store(pages: KvPages, k, v, off, start, table, status=None, stream=None) -> None:
    """New tokens into 8-bit blocks: rows k, v [rows, kv_heads, dim]; see include/netkv.h."""
    _kv_move("netkv_kv_store", _lib.netkv_kv_store, pages, k, v, off, start, table, status, stream)


def netkv_kv_load(pages: KvPages, k, v, off, start, table, status=None, stream=None) -> None:
    """Tokens from 8-bit blocks into the rows k, v; see include/netkv.h."""
    _kv_move("netkv_kv_load", _lib.netkv_kv_load, pages, k, v, off, start, table, status, stream)


def netkv_attn_prompt(q, k, v, q_off, k_off, out, lse=None, scale=None, status=None,
                      stream=None) -> None:
    """Causal attention of packed prompts: q, out [q_rows, heads, dim], k, v [k_rows, kv_heads,
    dim]; scale defaults to dim ** -0.5.  See include/netkv.h."""
    q_rows, heads, dim = q.shape
    k_rows, kv_heads, _ = k.shape
    d = _device(q)
    dt, qp, qs = _rows(q, heads, dim, d)
    _, kp, ks = _rows(k, kv_heads, dim, d, dt)
    _, vp, vs = _rows(v, kv_heads, dim, d, dt)
    _, op, os_ = _rows(out, heads, dim, d, dt)
    if v.shape[0] != k_rows or out.shape[0] != q_rows:
        raise ValueError("as many rows of keys as of values, and of out as of q, expected")
    n = q_off.numel() - 1
    _check("netkv_attn_prompt", _lib.netkv_attn_prompt(
        dt, qp, qs, kp, ks, vp, vs, heads, kv_heads, dim, n, _ints(q_off, _I64, n + 1, d),
        _ints(k_off, _I64, n + 1, d), q_rows, k_rows, dim ** -0.5 if scale is None else scale,
        op, os_, _plane(lse, q_rows, heads, d), _word(status, d), _on_stream(d, stream)))


def netkv_attn_decode_workspace_size(pages: KvPages, n_seqs: int, heads: int, table_width: int,
                                     with_mass: bool = False) -> int:
    """Bytes of the workspace; see include/netkv.h."""
    return int(_lib.netkv_attn_decode_workspace_size(pages.ref, int(n_seqs), int(heads),
                                                     int(table_width), int(bool(with_mass))))


def netkv_attn_decode(pages: KvPages, q, length, table, out, lse=None, mass_in=None, mass_out=None,
                      scale=None, workspace=None, status=None, stream=None) -> None:
    """One query row a sequence over its blocks: q, out [n_seqs, heads, dim]; see
    include/netkv.h."""
    n, heads, dim = q.shape
    d = _device(q)
    if pages.device_index != d:
        _elsewhere(pages, d)
    dt, qp, qs = _rows(q, heads, pages.heads_dim[1], d)
    _, op, os_ = _rows(out, heads, dim, d, dt)
    if out.shape[0] != n:
        raise ValueError("as many rows of out as of q expected")
    tp, tw = _table(table, n, d)
    wp, ws_bytes = None, 0
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("a contiguous workspace expected")
        if workspace.get_device() != d:
            _elsewhere(workspace, d)
        wp, ws_bytes = workspace.data_ptr(), workspace.nbytes
    _check("netkv_attn_decode", _lib.netkv_attn_decode(
        pages.ref, dt, qp, qs, heads, n, _ints(length, _I32, n, d), tp, tw,
        dim ** -0.5 if scale is None else scale, op, os_, _plane(lse, n, heads, d),
        _plane(mass_in, n, tw, d), _plane(mass_out, n, tw, d), wp, ws_bytes,
        _word(status, d), _on_stream(d, stream)))


def netkv_kv_evict(table, length, mass, budget, sink: int, recent: int, table_out, length_out,
                   mass_out, freed, n_freed, status=None, stream=None) -> None:
    """Block tables cut to a budget by accumulated attention weight; see include/netkv.h."""
    n = length.numel()
    d = _device(table)
    tp, tw = _table(table, n, d)
    to, two = _table(table_out, n, d)
    fr, twf = _table(freed, n, d)
    if two != tw or twf != tw:
        raise ValueError("tables of one width expected")
    _check("netkv_kv_evict", _lib.netkv_kv_evict(
        n, tp, _ints(length, _I32, n, d), _plane(mass, n, tw, d), tw, _ints(budget, _I32, n, d),
        int(sink), int(recent), to, _ints(length_out, _I32, n, d), _plane(mass_out, n, tw, d), fr,
        _ints(n_freed, _I32, n, d), _word(status, d), _on_stream(d, stream)))


def make_weights(w: np.ndarray, theta: float, cap_tokens: int, bytes_per_token: int) -> np.ndarray:
    """Host array of netkv_weights from an [n_streams, 3] (w_net, w_prefix, w_load) array."""
    w = np.asarray(w, dtype=np.float32).reshape(-1, 3)
    out = np.zeros(len(w), WEIGHTS_DTYPE)
    out["w_net"], out["w_prefix"], out["w_load"] = w[:, 0], w[:, 1], w[:, 2]
    out["theta_s_per_token"] = np.float32(theta)
    out["cap_tokens"] = int(cap_tokens)
    out["bytes_per_token"] = int(bytes_per_token)
    return out


def index_log2_capacity(max_distinct_keys: int) -> int:
    """Smallest table size keeping a cache-index table at load factor <= 0.5."""
    l = 1
    while (1 << l) < 2 * max(int(max_distinct_keys), 1):
        l += 1
    return l
