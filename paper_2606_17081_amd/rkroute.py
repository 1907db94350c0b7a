"""ctypes binding of ``librkroute.so`` (the C ABI in include/rkroute.h).

Argument marshalling only: every computation runs in the HIP library.  PyTorch
supplies device memory and the current stream.  Importing this module does
not need a GPU; calling a compute entry point without the built library or a
GPU raises immediately.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librkroute.so")

RK_OK, RK_EINVAL, RK_ENOMEM, RK_EHIP, RK_ETABLEFULL, RK_EUNSUPPORTED = 0, -1, -2, -3, -4, -5
RK_PROBE_PREFIX, RK_PROBE_SCAN = 0, 1
RK_POLICY_ARGMIN, RK_POLICY_SOFTMAX, RK_POLICY_ROUND_ROBIN, RK_POLICY_RANDOM, RK_POLICY_P2C = range(5)
RK_EVICT_LRU, RK_EVICT_FREQ = 0, 1
RK_FREQ_CAP = 1 << 20
DEV_BITS = {0x1: "bad offsets", 0x2: "short input", 0x4: "zero key", 0x8: "table full",
            0x10: "too large", 0x20: "no convergence", 0x40: "bad policy parameters", 0x80: "bad block"}
RK_BLOCK_TOKENS, RK_MAX_BATCH = 16, 4096
RK_BF16, RK_F16 = 0, 1

EXPORTED = ("rk_status_string", "rk_last_error", "rk_device_status", "rk_hash_chains",
            "rk_table_build", "rk_route_score_batch", "rk_index_build", "rk_route_score_index",
            "rk_simulate_workspace_size",
            "rk_simulate_episodes", "rk_poa_workspace_size", "rk_poa_estimate",
            "rk_poa_estimate_noalloc", "rk_prefix_groups", "rk_block_tables", "rk_kv_write",
            "rk_prefix_attention_workspace_size", "rk_prefix_attention", "rk_kv_write_fp4", "rk_kv_read_fp4",
            "rk_prefix_attention_fp4_workspace_size", "rk_prefix_attention_fp4")
RK_POA_NOALLOC_BYTES = 64 << 20


class RkError(RuntimeError):
    pass


class CostParams(C.Structure):
    _fields_ = [("w_ov", C.c_float), ("w_act", C.c_float), ("w_sat", C.c_float),
                ("cap_blocks", C.c_int32)]


class PoaParams(C.Structure):
    _fields_ = [("a", C.c_float), ("b", C.c_float), ("d", C.c_float), ("beta", C.c_int32),
                ("C_cap", C.c_int32), ("w_c", C.c_float), ("K_fixed", C.c_int32)]


class RegimeParams(C.Structure):
    _fields_ = [("alpha", C.c_double), ("theta1", C.c_double), ("theta2", C.c_double), ("eps", C.c_double),
                ("k", C.c_int32), ("beta", C.c_int32), ("a", C.c_double), ("b", C.c_double), ("d", C.c_double),
                ("n_sat", C.c_int32), ("tau", C.c_float * 3), ("w_ov", C.c_float * 3)]


def regime_params(r: dict) -> RegimeParams:
    return RegimeParams(r["alpha"], r["theta1"], r["theta2"], r["eps"], r["k"], r["beta"], r["a"], r["b"], r["d"],
                        r["n_sat"], (C.c_float * 3)(*r["tau"]), (C.c_float * 3)(*r["w_ov"]))


class EpisodeBatch(C.Structure):
    _fields_ = [("E", C.c_int32), ("W", C.c_int32), ("cache_blocks", C.c_int32),
                ("max_blocks", C.c_int32), ("max_conv", C.c_int32), ("max_inflight", C.c_int32),
                ("max_routes_per_step", C.c_int32), ("max_ctrl_window", C.c_int32),
                ("probe_mode", C.c_int32), ("tiers", C.c_int32), ("max_routes", C.c_int32),
                ("flags", C.c_int32), ("ws_slots", C.c_int32), ("ws_pad", C.c_int32),
                ("params", C.c_void_p), ("turn_off", C.c_void_p), ("turn_blocks", C.c_void_p),
                ("chain_off", C.c_void_p), ("chains", C.c_void_p), ("route_rand", C.c_void_p),
                ("regime", RegimeParams)]


class EpisodeOutputs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("route_turn", "route_worker", "route_step", "route_blocks",
                                          "overlap", "cost", "evict_count", "evict_digest",
                                          "last_hash", "totals", "route_regime", "tier_overlap")]


class CacheStrides(C.Structure):
    _fields_ = [("block", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class Attention(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32),
                ("n_blocks", C.c_int32), ("table_stride", C.c_int32), ("scale", C.c_float), ("T", C.c_int64),
                ("q", C.c_void_p), ("q_token", C.c_int64), ("q_head", C.c_int64),
                ("k_cache", C.c_void_p), ("ks", CacheStrides), ("v_cache", C.c_void_p), ("vs", CacheStrides),
                ("tables", C.c_void_p), ("kv_len", C.c_void_p), ("q_off", C.c_void_p),
                ("group_off", C.c_void_p), ("shared", C.c_void_p),
                ("out", C.c_void_p), ("out_token", C.c_int64), ("out_head", C.c_int64), ("lse", C.c_void_p)]


class Fp4Cache(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("cs", CacheStrides), ("scales", C.c_void_p), ("ss", CacheStrides)]


class AttentionFp4(C.Structure):
    _fields_ = [("a", Attention), ("k", Fp4Cache), ("v", Fp4Cache)]


# rk_episode_params, 104 bytes, as a numpy record
EPISODE_PARAMS_DTYPE = np.dtype([
    ("conv_begin", "<i8"), ("n_conv", "<i4"), ("hold_steps", "<i4"), ("routes_per_step", "<i4"),
    ("controller", "<i4"), ("ctrl_window", "<i4"), ("ctrl_num", "<i4"), ("ctrl_den", "<i4"),
    ("cap_blocks", "<i4"), ("w_ov", "<f4"), ("w_act", "<f4"), ("w_sat", "<f4"),
    ("ctrl_w_ov", "<f4"), ("out_base", "<i8"), ("policy", "<i4"), ("tau", "<f4"),
    ("evict_policy", "<i4"), ("decay_steps", "<i4"), ("tier_g1", "<i4"), ("tier_g2", "<i4"),
    ("tier_w", "<f4", (3,)), ("tier_pad", "<i4")])
assert EPISODE_PARAMS_DTYPE.itemsize == 104

_lock = threading.Lock()
_lib = None


def library_available() -> bool:
    return os.path.exists(LIB_PATH)


def lib():
    """Load librkroute.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RkError(f"{LIB_PATH} is missing: build it with `python -m paper_2606_17081_amd.build`")
            L = C.CDLL(LIB_PATH)
            vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
            L.rk_status_string.restype = C.c_char_p
            L.rk_status_string.argtypes = [C.c_int]
            L.rk_last_error.restype = C.c_char_p
            L.rk_last_error.argtypes = []
            L.rk_device_status.restype = C.c_int
            L.rk_device_status.argtypes = [C.c_int, vp, vp]
            L.rk_hash_chains.restype = C.c_int
            L.rk_hash_chains.argtypes = [i64, vp, vp, vp, vp, vp]
            L.rk_table_build.restype = C.c_int
            L.rk_table_build.argtypes = [i32, vp, vp, vp, i32, vp]
            L.rk_route_score_batch.restype = C.c_int
            L.rk_route_score_batch.argtypes = [i32, i32, vp, vp, vp, i32, vp, CostParams, i32, vp, vp, vp, vp]
            L.rk_index_build.restype = C.c_int
            L.rk_index_build.argtypes = [i32, vp, vp, vp, i32, vp]
            L.rk_route_score_index.restype = C.c_int
            L.rk_route_score_index.argtypes = [i32, i32, vp, vp, vp, i32, vp, CostParams, i32, vp, vp, vp, vp]
            L.rk_simulate_workspace_size.restype = sz
            L.rk_simulate_workspace_size.argtypes = [i32, i32, i32, i32, i32, i32]
            L.rk_simulate_episodes.restype = C.c_int
            L.rk_simulate_episodes.argtypes = [C.POINTER(EpisodeBatch), C.POINTER(EpisodeOutputs), vp, sz, vp]
            L.rk_poa_workspace_size.restype = sz
            L.rk_poa_workspace_size.argtypes = [i64, i32]
            L.rk_poa_estimate.restype = C.c_int
            L.rk_poa_estimate.argtypes = [i32, vp, i32, vp, i64, i32, i32, vp, vp, vp, PoaParams,
                                          vp, vp, vp, vp, sz, vp]
            L.rk_poa_estimate_noalloc.restype = C.c_int
            L.rk_poa_estimate_noalloc.argtypes = [i32, vp, i32, vp, i64, i32, i32, vp, vp, vp, PoaParams,
                                                  vp, vp, vp, vp]
            L.rk_prefix_groups.restype = C.c_int
            L.rk_prefix_groups.argtypes = [i32, vp, vp, i32, vp, vp, vp, vp, vp]
            L.rk_block_tables.restype = C.c_int
            L.rk_block_tables.argtypes = [i32, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp, i64, vp, vp, vp]
            L.rk_kv_write.restype = C.c_int
            L.rk_kv_write.argtypes = [i64, i32, i32, vp, i64, i64, vp, i64, i64, vp, CacheStrides, vp, CacheStrides,
                                      i32, vp, vp]
            L.rk_prefix_attention_workspace_size.restype = sz
            L.rk_prefix_attention_workspace_size.argtypes = [i64, i32, i32, i32, i32]
            L.rk_prefix_attention.restype = C.c_int
            L.rk_prefix_attention.argtypes = [vp, vp, sz, vp]
            L.rk_kv_write_fp4.restype = C.c_int
            L.rk_kv_write_fp4.argtypes = [i64, i32, i32, i32, vp, i64, i64, vp, i64, i64, vp, vp, i32, vp, vp]
            L.rk_kv_read_fp4.restype = C.c_int
            L.rk_kv_read_fp4.argtypes = [i64, i32, i32, i32, vp, vp, i32, vp, vp, i64, i64, vp, i64, i64, vp]
            L.rk_prefix_attention_fp4_workspace_size.restype = sz
            L.rk_prefix_attention_fp4_workspace_size.argtypes = [i64, i32, i32, i32, i32]
            L.rk_prefix_attention_fp4.restype = C.c_int
            L.rk_prefix_attention_fp4.argtypes = [vp, vp, sz, vp]
            _lib = L
    return _lib


def _check(rc: int, what: str):
    if rc != RK_OK:
        L = lib()
        raise RkError(f"{what}: {L.rk_status_string(rc).decode()} ({rc}): {L.rk_last_error().decode()}")


_found_torch = None


def _torch():
    """torch, once it has seen a GPU (asking again costs microseconds, several times a call)."""
    global _found_torch
    if _found_torch is None:
        import torch
        if not torch.cuda.is_available():
            raise RkError("no GPU visible: the routing library runs on an MI355X (gfx950) device only")
        _found_torch = torch
    return _found_torch


def _ptr(t) -> Optional[int]:
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    torch = _torch()
    if stream is not None:
        return C.c_void_p(stream.cuda_stream)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)    # the handle without a Stream object
    return C.c_void_p(raw(torch.cuda.current_device()) if raw else torch.cuda.current_stream().cuda_stream)


def _need(t, dtype, name):
    torch = _torch()
    if t is None:
        return
    ok = (torch.int64, torch.uint64) if dtype in (torch.int64, torch.uint64) and name in _HASH_ARGS else (dtype,)
    if not t.is_cuda or t.dtype not in ok or not t.is_contiguous():
        raise RkError(f"{name} must be a contiguous CUDA tensor of {dtype}")


def _outputs_fit(B, W, overlap, cost, argmin):
    for t, n, name in ((overlap, B * W, "overlap"), (cost, B * W, "cost"), (argmin, B, "argmin")):
        if t is not None and t.numel() < n:
            raise RkError(f"{name} holds {t.numel()} elements, {n} needed")


# 64-bit block hashes may live in int64 tensors (same bits; PyTorch supports
# more int64 operations than uint64 ones).
_HASH_ARGS = ("chains", "keys", "tables", "index", "evict_digest", "last_hash")


def to_device(a: np.ndarray, device="cuda"):
    """Upload a numpy array; uint64 arrays become int64 tensors with the same bits."""
    torch = _torch()
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint64:
        a = a.view(np.int64)
    return torch.from_numpy(a).to(device)


def to_host_u64(t) -> np.ndarray:
    """Copy a 64-bit hash tensor back as uint64."""
    return t.cpu().numpy().view(np.uint64)


# ------------------------------------------------------------------ entry points

def device_status(reset: bool = True, stream=None) -> int:
    bits = np.zeros(1, np.int32)
    _check(lib().rk_device_status(int(reset), C.c_void_p(bits.ctypes.data), _stream(stream)),
           "rk_device_status")
    return int(bits[0])


def hash_chains(tokens, tok_off, chain_off, chains=None, stream=None):
    """Block-hash chains of token sequences (see rk_hash_chains)."""
    torch = _torch()
    _need(tokens, torch.int32, "tokens")
    _need(tok_off, torch.int64, "tok_off")
    _need(chain_off, torch.int64, "chain_off")
    n_seq = tok_off.numel() - 1
    if chains is None:
        n = int(chain_off[-1].item()) if n_seq > 0 else 0
        chains = torch.empty(max(n, 1), dtype=torch.int64, device=tokens.device)
    _need(chains, torch.uint64, "chains")
    _check(lib().rk_hash_chains(n_seq, _ptr(tokens), _ptr(tok_off), _ptr(chain_off), _ptr(chains),
                                _stream(stream)), "rk_hash_chains")
    return chains


def table_build(keys, key_off: np.ndarray, log2_slots: int, tables=None, stream=None):
    """W open-addressing tables from per-worker key lists (key_off is a host array)."""
    torch = _torch()
    _need(keys, torch.uint64, "keys")
    key_off = np.ascontiguousarray(key_off, dtype=np.int64)
    W = key_off.shape[0] - 1
    if tables is None:
        tables = torch.empty(W << log2_slots, dtype=torch.int64, device=keys.device)
    _need(tables, torch.uint64, "tables")
    _check(lib().rk_table_build(W, _ptr(keys), C.c_void_p(key_off.ctypes.data), _ptr(tables), log2_slots,
                                _stream(stream)), "rk_table_build")
    return tables


def route_score_batch(chains, chain_off, tables, log2_slots: int, active_blocks, w_ov=1.0, w_act=0.5,
                      w_sat=4.0, cap_blocks=32768, probe_mode=RK_PROBE_PREFIX, overlap=None, cost=None,
                      argmin=None, want_overlap=True, want_cost=True, stream=None):
    """Overlap and cost per (request, worker) and argmin per request."""
    torch = _torch()
    _need(chains, torch.uint64, "chains")
    _need(chain_off, torch.int64, "chain_off")
    _need(tables, torch.uint64, "tables")
    _need(active_blocks, torch.int32, "active_blocks")
    B = chain_off.numel() - 1
    W = active_blocks.numel()
    dev = chains.device
    if overlap is None and want_overlap:
        overlap = torch.empty((B, W), dtype=torch.int32, device=dev)
    if cost is None and want_cost:
        cost = torch.empty((B, W), dtype=torch.float32, device=dev)
    if argmin is None:
        argmin = torch.empty(B, dtype=torch.int32, device=dev)
    _need(overlap, torch.int32, "overlap")
    _need(cost, torch.float32, "cost")
    _need(argmin, torch.int32, "argmin")
    _outputs_fit(B, W, overlap, cost, argmin)
    p = CostParams(w_ov, w_act, w_sat, cap_blocks)
    _check(lib().rk_route_score_batch(B, W, _ptr(chains), _ptr(chain_off), _ptr(tables), log2_slots,
                                      _ptr(active_blocks), p, probe_mode, _ptr(overlap), _ptr(cost),
                                      _ptr(argmin), _stream(stream)), "rk_route_score_batch")
    return overlap, cost, argmin


def index_build(keys, key_off: np.ndarray, log2_slots: int, index=None, stream=None):
    """The global block index (key, worker mask) over W workers' key lists
    (key_off is a host array); 16-byte slots held as int64 pairs."""
    torch = _torch()
    _need(keys, torch.uint64, "keys")
    key_off = np.ascontiguousarray(key_off, dtype=np.int64)
    W = key_off.shape[0] - 1
    if index is None:
        index = torch.empty(2 << log2_slots, dtype=torch.int64, device=keys.device)
    _need(index, torch.uint64, "index")
    if index.numel() < (2 << log2_slots):
        raise RkError("index holds fewer than 2^log2_slots 16-byte slots")
    _check(lib().rk_index_build(W, _ptr(keys), C.c_void_p(key_off.ctypes.data), _ptr(index), log2_slots,
                                _stream(stream)), "rk_index_build")
    return index


def route_score_index(chains, chain_off, index, log2_slots: int, active_blocks, w_ov=1.0, w_act=0.5,
                      w_sat=4.0, cap_blocks=32768, probe_mode=RK_PROBE_PREFIX, overlap=None, cost=None,
                      argmin=None, want_overlap=True, want_cost=True, stream=None):
    """route_score_batch against the global block index (rk_route_score_index)."""
    torch = _torch()
    _need(chains, torch.uint64, "chains")
    _need(chain_off, torch.int64, "chain_off")
    _need(index, torch.uint64, "index")
    _need(active_blocks, torch.int32, "active_blocks")
    B = chain_off.numel() - 1
    W = active_blocks.numel()
    if index.numel() < (2 << log2_slots):
        raise RkError("index holds fewer than 2^log2_slots 16-byte slots")
    dev = chains.device
    if overlap is None and want_overlap:
        overlap = torch.empty((B, W), dtype=torch.int32, device=dev)
    if cost is None and want_cost:
        cost = torch.empty((B, W), dtype=torch.float32, device=dev)
    if argmin is None:
        argmin = torch.empty(B, dtype=torch.int32, device=dev)
    _need(overlap, torch.int32, "overlap")
    _need(cost, torch.float32, "cost")
    _need(argmin, torch.int32, "argmin")
    _outputs_fit(B, W, overlap, cost, argmin)
    p = CostParams(w_ov, w_act, w_sat, cap_blocks)
    _check(lib().rk_route_score_index(B, W, _ptr(chains), _ptr(chain_off), _ptr(index), log2_slots,
                                      _ptr(active_blocks), p, probe_mode, _ptr(overlap), _ptr(cost),
                                      _ptr(argmin), _stream(stream)), "rk_route_score_index")
    return overlap, cost, argmin


def simulate_workspace_size(E, W, cache_blocks, max_blocks, max_conv, max_routes) -> int:
    return int(lib().rk_simulate_workspace_size(E, W, cache_blocks, max_blocks, max_conv, max_routes))


def simulate_episodes(batch: EpisodeBatch, outputs: EpisodeOutputs, workspace, stream=None):
    """Launch rk_simulate_episodes on prepared structs (see EpisodeRunner for the usual path)."""
    _check(lib().rk_simulate_episodes(C.byref(batch), C.byref(outputs), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream(stream)),
           "rk_simulate_episodes")


def poa_workspace_size(n_rows: int, W: int) -> int:
    return int(lib().rk_poa_workspace_size(n_rows, W))


def poa_estimate(win_off, ep_win_off, n_rows: int, max_window: int, W: int, route_worker, overlap,
                 route_blocks, params: PoaParams, selfish, coord, poa_hat, workspace, stream=None):
    n_windows = win_off.numel() - 1
    n_eps = 0 if ep_win_off is None else ep_win_off.numel() - 1
    _check(lib().rk_poa_estimate(n_windows, _ptr(win_off), n_eps, _ptr(ep_win_off), n_rows, max_window, W,
                                 _ptr(route_worker), _ptr(overlap), _ptr(route_blocks), params,
                                 _ptr(selfish), _ptr(coord), _ptr(poa_hat), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)),
           "rk_poa_estimate")


def poa_estimate_noalloc(win_off, ep_win_off, n_rows: int, max_window: int, W: int, route_worker, overlap,
                         route_blocks, params: PoaParams, selfish, coord, poa_hat, stream=None):
    """poa_estimate on the library's static device buffer (rk_poa_estimate_noalloc):
    no workspace argument, nothing allocated by the call."""
    n_windows = win_off.numel() - 1
    n_eps = 0 if ep_win_off is None else ep_win_off.numel() - 1
    _check(lib().rk_poa_estimate_noalloc(n_windows, _ptr(win_off), n_eps, _ptr(ep_win_off), n_rows, max_window, W,
                                         _ptr(route_worker), _ptr(overlap), _ptr(route_blocks), params,
                                         _ptr(selfish), _ptr(coord), _ptr(poa_hat), _stream(stream)),
           "rk_poa_estimate_noalloc")


# ------------------------------------------------------------------ a worker's step
#
# These run once or more per layer of a model on batches that take the GPU microseconds, so a call's own time counts: checks go
# by device numbers and stride tuples, and arguments are passed as plain numbers.

_NARROW = {}                                   # names of 16-bit types, filled with torch


def _where(name, t):
    """The number of the GPU that holds t."""
    dev = t.get_device()
    if dev < 0:
        _torch()
        raise RkError(f"{name} must be a CUDA tensor")
    return dev


class _On:
    """Where a call with tensors on GPU `dev` runs: on the given stream, or on that GPU's current one (both as the raw
    handle).  Meanwhile it is the current stream, so that what the call allocates is that stream's too."""
    __slots__ = ("context", "dev")

    def __init__(self, dev, stream):
        torch = _found_torch or _torch()
        self.dev, self.context = dev, None
        if stream is not None:
            if stream.device.index != dev:
                raise RkError(f"the stream is on {stream.device}, the tensors are on cuda:{dev}")
            self.context = torch.cuda.stream(stream)
        elif torch._C._cuda_getDevice() != dev:
            self.context = torch.cuda.device(dev)

    def __enter__(self):
        if self.context is not None:
            self.context.__enter__()
        return _found_torch._C._cuda_getCurrentRawStream(self.dev)

    def __exit__(self, *exc):
        if self.context is not None:
            self.context.__exit__(*exc)
        return False


def _flat(name, t, dtype, dev, n):
    """The address of a contiguous tensor of at least n elements (None: of none)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise RkError(f"{name} is on {t.device}, not on cuda:{dev}")
    if t.dtype != dtype or not t.is_contiguous():
        if not (name in _HASH_ARGS and t.dtype == _found_torch.uint64 and t.is_contiguous()):
            raise RkError(f"{name} must be a contiguous CUDA tensor of {dtype}")
    if t.numel() < n:
        raise RkError(f"{name} holds {t.numel()} elements, {n} needed")
    return t.data_ptr()


def _changed(*tensors):
    """Counts a write for autograd, to which the library's are not visible: a backward pass that saved such a tensor is to say so.
    (None: none.)"""
    _found_torch.autograd.graph.increment_version([t for t in tensors if t is not None])


def prefix_groups(chains, chain_off, min_blocks: int = 1, order=None, group_off=None, shared=None, n_groups=None,
                  stream=None):
    """The batch ordered by shared prompt prefix (rk_prefix_groups): (order, group_off, shared, n_groups)."""
    dev = _where("chain_off", chain_off)
    with _On(dev, stream) as st:
        torch = _found_torch
        i32, i64 = torch.int32, torch.int64
        B = chain_off.numel() - 1
        if B < 0:
            raise RkError("chain_off is empty")
        at = chain_off.device
        given = order, group_off, shared, n_groups
        if order is None:
            order = torch.empty(B, dtype=i32, device=at)
        if group_off is None:
            group_off = torch.empty(B + 1, dtype=i64, device=at)
        if shared is None:
            shared = torch.empty(B, dtype=i32, device=at)
        if n_groups is None:
            n_groups = torch.empty(1, dtype=i32, device=at)
        _check(lib().rk_prefix_groups(
            B, _flat("chains", chains, i64, dev, 0), _flat("chain_off", chain_off, i64, dev, 0), min_blocks,
            _flat("order", order, i32, dev, B), _flat("group_off", group_off, i64, dev, B + 1),
            _flat("shared", shared, i32, dev, B), _flat("n_groups", n_groups, i32, dev, 1), st), "rk_prefix_groups")
        _changed(*given)
    return order, group_off, shared, n_groups


def block_tables(tables, kv_len, new_len, have, free_blocks, n_slots: int, group_off=None, shared=None, slots=None,
                 q_off=None, taken=None, stream=None):
    """Block tables (in place) and slot map of a step (rk_block_tables): (tables, slots, q_off, taken).
    tables is [B, stride]; n_slots is the number of slots wanted, the step's new tokens or more."""
    dev = _where("kv_len", kv_len)
    with _On(dev, stream) as st:
        torch = _found_torch
        i32, i64 = torch.int32, torch.int64
        B, at = kv_len.numel(), kv_len.device
        rows, stride = _table_shape(tables, B)
        given = tables, slots, q_off, taken
        if slots is None:
            slots = torch.empty(n_slots, dtype=i64, device=at)
        if q_off is None:
            q_off = torch.empty(B + 1, dtype=i64, device=at)
        if taken is None:
            taken = torch.empty(1, dtype=i32, device=at)
        _check(lib().rk_block_tables(
            B, _flat("kv_len", kv_len, i32, dev, B), _flat("new_len", new_len, i32, dev, B),
            _flat("have", have, i32, dev, B), _flat("group_off", group_off, i64, dev, B + 1),
            _flat("shared", shared, i32, dev, B), _flat("free_blocks", free_blocks, i32, dev, 0), free_blocks.numel(),
            _flat("tables", tables, i32, dev, 0), stride, _flat("slots", slots, i64, dev, n_slots), n_slots,
            _flat("q_off", q_off, i64, dev, B + 1), _flat("taken", taken, i32, dev, 1), st), "rk_block_tables")
        _changed(*given)
    return tables, slots, q_off, taken


def _table_shape(tables, B):
    shape = tables.shape
    if len(shape) != 2 or shape[0] < B:
        raise RkError("tables must be [B, stride]")
    return shape


def _rows(name, t, dev, dtype, shape):
    """The strides of tokens and heads of a [tokens, heads, D] tensor with its heads' elements side by side."""
    if t.get_device() != dev or t.dtype != dtype:
        raise RkError(f"{name} must be a tensor of {dtype} on cuda:{dev}")
    if t.shape != shape:
        raise RkError(f"{name} must be {list(shape)}, it is {list(t.shape)}")
    token, head, one = t.stride()
    if one != 1 and t.numel():
        raise RkError(f"{name} must have a head's elements side by side")
    return token if shape[0] > 1 else 0, head if shape[0] and shape[1] > 1 else 0      # of one, any stride will do


_strides_made = {}


def _cache_strides(name, t, dev, dtype, shape):
    if t.get_device() != dev or t.dtype != dtype:
        raise RkError(f"{name} must be a tensor of {dtype} on cuda:{dev}")
    if t.shape != shape:
        raise RkError(f"{name} must be {list(shape)}, it is {list(t.shape)}")
    block, token, head, one = t.stride()
    if not t.numel():
        block, token, head = 0, shape[3], 0
    elif one != 1:
        raise RkError(f"{name} must have a head's elements side by side")
    return block if shape[0] > 1 else 0, token, head if shape[2] > 1 else 0


def _as_strides(s):
    """The three strides as the ABI's struct (made once for each, and never written)."""
    got = _strides_made.get(s)
    if got is None:
        if len(_strides_made) > 256:
            _strides_made.clear()
        got = _strides_made[s] = CacheStrides(*s)
    return got


def _heads(name, t, dims):
    """dtype and shape of a tensor of 16-bit floating values."""
    if not _NARROW:
        torch = _torch()
        _NARROW.update({torch.bfloat16: RK_BF16, torch.float16: RK_F16})
    if t.dtype not in _NARROW or t.dim() != dims:
        raise RkError(f"{name} must be a CUDA tensor of bfloat16 or float16 with {dims} dimensions")
    return t.dtype, t.shape


def _no_gradient(what, *tensors):
    """Refuses tensors whose gradient, or forward-mode tangent, a call would drop (None: no tensor)."""
    torch = _found_torch or _torch()
    forward = torch.autograd.forward_ad
    for t in tensors:
        if t is None:
            continue
        if t.requires_grad and torch.is_grad_enabled():
            raise RkError(f"{what} has no gradient: call it under torch.no_grad(), or detach its arguments")
        if forward._current_level >= 0 and forward.unpack_dual(t).tangent is not None:
            raise RkError(f"{what} has no forward-mode derivative: call it on the primal tensors")


def kv_write(k, v, k_cache, v_cache, slots, stream=None):
    """Keys and values [T, Hkv, D] of new tokens into the block cache [blocks, 16, Hkv, D] (rk_kv_write)."""
    dev = _where("k", k)
    _no_gradient("kv_write", k, v, k_cache, v_cache)
    dtype, shape = _heads("k", k, 3)
    T, Hkv, D = shape
    k_token, k_head = _rows("k", k, dev, dtype, shape)
    v_token, v_head = _rows("v", v, dev, dtype, shape)
    if k_cache.dim() != 4:
        raise RkError("k_cache must be [blocks, 16, heads, D]")
    blocks = k_cache.shape[0]
    cache = (blocks, RK_BLOCK_TOKENS, Hkv, D)
    ks = _as_strides(_cache_strides("k_cache", k_cache, dev, dtype, cache))
    vs = _as_strides(_cache_strides("v_cache", v_cache, dev, dtype, cache))
    with _On(dev, stream) as st:
        _check(lib().rk_kv_write(T, Hkv, D, k.data_ptr(), k_token, k_head, v.data_ptr(), v_token, v_head,
                                 k_cache.data_ptr(), ks, v_cache.data_ptr(), vs, blocks,
                                 _flat("slots", slots, _found_torch.int64, dev, T), st), "rk_kv_write")
        _changed(k_cache, v_cache)


def prefix_attention_workspace_size(T: int, B: int, Hq: int, Hkv: int, D: int) -> int:
    """Bytes of workspace for T tokens of B requests in groups; for T = 0, of any number of tokens without groups."""
    return int(lib().rk_prefix_attention_workspace_size(T, B, Hq, Hkv, D))


_attention_struct = struct.Struct("@7ifq" + "P2q" + "P3qP3q" + "5P" + "P2qP")
assert _attention_struct.size == C.sizeof(Attention)


def prefix_attention(q, k_cache, v_cache, tables, kv_len, q_off, group_off=None, shared=None, scale=None, out=None,
                     lse=None, want_lse=False, workspace=None, stream=None):
    """Attention of new tokens q [T, Hq, D] over the block cache (rk_prefix_attention): (out, lse or None).
    scale defaults to D ** -0.5.  Rows behind the last request's stay as they were (in an `out` allocated here,
    uninitialised)."""
    dev = _where("q", q)
    _no_gradient("prefix_attention", q, k_cache, v_cache, out, lse)
    dtype, shape = _heads("q", q, 3)
    if k_cache.dim() != 4:
        raise RkError("k_cache must be [blocks, 16, heads, D]")
    blocks, _, Hkv, _ = k_cache.shape
    cache = (blocks, RK_BLOCK_TOKENS, Hkv, shape[2])
    ks = _cache_strides("k_cache", k_cache, dev, dtype, cache)
    vs = _cache_strides("v_cache", v_cache, dev, dtype, cache)
    return _attend("rk_prefix_attention", dev, q, dtype, shape, blocks, Hkv, (k_cache.data_ptr(), *ks, v_cache.data_ptr(), *vs),
                   b"", tables, kv_len, q_off, group_off, shared, scale, out, lse, want_lse, workspace, stream)


def _attend(name, dev, q, dtype, shape, blocks, Hkv, caches, more, tables, kv_len, q_off, group_off, shared, scale, out, lse,
            want_lse, workspace, stream):
    """The call `name`; caches: pointers and strides of 16-bit caches, more: what follows the rk_attention."""
    T, Hq, D = shape
    q_token, q_head = _rows("q", q, dev, dtype, shape)
    with _On(dev, stream) as st:
        torch = _found_torch
        i32, i64 = torch.int32, torch.int64
        B, at = kv_len.numel(), q.device
        _, stride = _table_shape(tables, B)
        given = [t for t in (out, lse) if t is not None]
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=at)
            out_token, out_head = Hq * D, D
        else:
            out_token, out_head = _rows("out", out, dev, dtype, shape)
        if lse is None and want_lse:
            lse = torch.empty((T, Hq), dtype=torch.float32, device=at)
        L = lib()
        if workspace is None:
            ws_bytes = getattr(L, name + "_workspace_size")(T if group_off is not None else 0, B, Hq, Hkv, D)
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=at)
        elif workspace.get_device() != dev or not workspace.is_contiguous():
            raise RkError(f"workspace must be a contiguous tensor on cuda:{dev}")
        else:
            ws_bytes = workspace.numel() * workspace.element_size()
        a = _attention_struct.pack(
            B, Hq, Hkv, D, _NARROW[dtype], blocks, stride, max(D, 1) ** -0.5 if scale is None else scale, T, q.data_ptr(),
            q_token, q_head, *caches, _flat("tables", tables, i32, dev, 0),
            _flat("kv_len", kv_len, i32, dev, B), _flat("q_off", q_off, i64, dev, B + 1),
            _flat("group_off", group_off, i64, dev, B + 1) or 0, _flat("shared", shared, i32, dev, B) or 0,
            out.data_ptr(), out_token, out_head, _flat("lse", lse, torch.float32, dev, T * Hq) or 0) + more
        _check(getattr(L, name)(a, workspace.data_ptr(), ws_bytes, st), name)
        if given:
            _changed(*given)
    return out, lse


# ------------------------------------------------------------------ a worker's cache in 4 bits

_fp4_struct = struct.Struct("@P3qP3q")
assert _fp4_struct.size == C.sizeof(Fp4Cache) and C.sizeof(AttentionFp4) == _attention_struct.size + 2 * _fp4_struct.size


def _fp4_cache(which, codes, scales, dev, blocks, Hkv, D):
    """A cache in 4 bits as the ABI's struct: codes [blocks, 16, Hkv, 16 C], scales [blocks, 16, Hkv, C], C = ceil(D / 32)."""
    u8, C_ = _found_torch.uint8, -(-D // 32)
    shape = (blocks, RK_BLOCK_TOKENS, Hkv)
    return _fp4_struct.pack(codes.data_ptr(), *_cache_strides(which + "_cache", codes, dev, u8, (*shape, 16 * C_)),
                            scales.data_ptr(), *_cache_strides(which + "_scales", scales, dev, u8, (*shape, C_)))


def kv_write_fp4(k, v, k_cache, v_cache, k_scales, v_scales, slots, stream=None):
    """Keys and values [T, Hkv, D] of new tokens into a cache in 4 bits (rk_kv_write_fp4): codes uint8 [blocks, 16, Hkv, 16 C],
    scales uint8 [blocks, 16, Hkv, C], C = ceil(D / 32)."""
    dev = _where("k", k)
    _no_gradient("kv_write_fp4", k, v)
    dtype, shape = _heads("k", k, 3)
    T, Hkv, D = shape
    k_token, k_head = _rows("k", k, dev, dtype, shape)
    v_token, v_head = _rows("v", v, dev, dtype, shape)
    if k_cache.dim() != 4:
        raise RkError("k_cache must be [blocks, 16, heads, 16 ceil(D / 32)]")
    blocks = k_cache.shape[0]
    kc, vc = _fp4_cache("k", k_cache, k_scales, dev, blocks, Hkv, D), _fp4_cache("v", v_cache, v_scales, dev, blocks, Hkv, D)
    with _On(dev, stream) as st:
        _check(lib().rk_kv_write_fp4(T, Hkv, D, _NARROW[dtype], k.data_ptr(), k_token, k_head, v.data_ptr(), v_token, v_head, kc, vc,
                                     blocks, _flat("slots", slots, _found_torch.int64, dev, T), st), "rk_kv_write_fp4")
        _changed(k_cache, v_cache, k_scales, v_scales)


def kv_read_fp4(k_cache, v_cache, k_scales, v_scales, slots, D=None, dtype=None, k=None, v=None, stream=None):
    """Tokens of a cache in 4 bits as 16-bit values (rk_kv_read_fp4): (k, v), [tokens, Hkv, D] each.  D defaults to the k that is
    given, or to all values of a row of codes (32 C); dtype to the k that is given, or to bfloat16."""
    dev = _where("k_cache", k_cache)
    torch = _found_torch or _torch()
    _no_gradient("kv_read_fp4", k, v)
    if k_cache.dim() != 4:
        raise RkError("k_cache must be [blocks, 16, heads, 16 ceil(D / 32)]")
    blocks, _, Hkv, row = k_cache.shape
    T = slots.numel()
    given = [t for t in (k, v) if t is not None]
    if D is None:
        D = 2 * row if not given else given[0].shape[-1]
    if dtype is None:
        dtype = given[0].dtype if given else torch.bfloat16
    with _On(dev, stream) as st:
        shape = (T, Hkv, D)
        if k is None:
            k = torch.empty(shape, dtype=dtype, device=k_cache.device)
        if v is None:
            v = torch.empty(shape, dtype=dtype, device=k_cache.device)
        _heads("k", k, 3)
        k_token, k_head = _rows("k", k, dev, dtype, shape)
        v_token, v_head = _rows("v", v, dev, dtype, shape)
        kc, vc = _fp4_cache("k", k_cache, k_scales, dev, blocks, Hkv, D), _fp4_cache("v", v_cache, v_scales, dev, blocks, Hkv, D)
        _check(lib().rk_kv_read_fp4(T, Hkv, D, _NARROW[dtype], kc, vc, blocks, _flat("slots", slots, torch.int64, dev, T),
                                    k.data_ptr(), k_token, k_head, v.data_ptr(), v_token, v_head, st), "rk_kv_read_fp4")
        if given:
            _changed(*given)
    return k, v


def prefix_attention_fp4_workspace_size(T: int, B: int, Hq: int, Hkv: int, D: int) -> int:
    """As prefix_attention_workspace_size, of prefix_attention_fp4."""
    return int(lib().rk_prefix_attention_fp4_workspace_size(T, B, Hq, Hkv, D))


def prefix_attention_fp4(q, k_cache, v_cache, k_scales, v_scales, tables, kv_len, q_off, group_off=None, shared=None, scale=None,
                         out=None, lse=None, want_lse=False, workspace=None, stream=None):
    """prefix_attention over a cache in 4 bits (rk_prefix_attention_fp4): (out, lse or None)."""
    dev = _where("q", q)
    _no_gradient("prefix_attention_fp4", q, out, lse)
    dtype, shape = _heads("q", q, 3)
    if k_cache.dim() != 4:
        raise RkError("k_cache must be [blocks, 16, heads, 16 ceil(D / 32)]")
    blocks, _, Hkv, _ = k_cache.shape
    more = (_fp4_cache("k", k_cache, k_scales, dev, blocks, Hkv, shape[2]) +
            _fp4_cache("v", v_cache, v_scales, dev, blocks, Hkv, shape[2]))
    return _attend("rk_prefix_attention_fp4", dev, q, dtype, shape, blocks, Hkv, (0,) * 8, more, tables, kv_len, q_off, group_off,
                   shared, scale, out, lse, want_lse, workspace, stream)
