"""Binding of libpikv.so: same names and argument order as include/pikv.h.

Every function takes torch tensors that already live in device memory (or None for
optional pointers), passes their addresses and the current HIP stream through the C ABI,
and returns nothing but the status check.  No arithmetic happens here.

The calls of a step are made by the extension _pikv_native (csrc/pikv_binding.cpp): eager passes over small caches are bound
by their calls, and ctypes with its attribute lookups took 4 - 5 us of each.  Arguments that are not of the ordinary kind -
tensor subclasses, numpy numbers, what has to be refused - come back from it as None with nothing launched and take the
ctypes path below, and so does every call where the extension is not there.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libpikv.so")
_NATIVE_PATH = os.path.join(_HERE, "_pikv_native.so")

F32, BF16 = 0, 1
COMBINE_LSE, COMBINE_LOCAL = 0, 1
PENALTY_LOAD_BALANCE, PENALTY_CACHE_AWARE, PENALTY_ENTROPY = 0, 1, 2
DESC_VALUE_BIAS, DESC_8BIT = 1, 2
POLICY_H2O, POLICY_SL, POLICY_LRU, POLICY_LRU_PLUS = 0, 1, 2, 3
QUANT_INT8, QUANT_E4M3 = 0, 1

EXPORTS = ("pikv_route", "pikv_attn_workspace_bytes", "pikv_sharded_attn", "pikv_update_utility",
           "pikv_evict", "pikv_append", "pikv_strerror", "pikv_version", "pikv_set_attn_split", "pikv_decode_step",
           "pikv_stream_read_probe",
           "pikv_set_profile_events", "pikv_router_penalty", "pikv_compress", "pikv_policy_stamp",
           "pikv_update_utility_tracked", "pikv_policy_utility", "pikv_policy_compact", "pikv_decode_step_policy", "pikv_route_round_robin",
           "pikv_sharded_attn_noalloc", "pikv_norm_rope", "pikv_quant_pack", "pikv_quant_read", "pikv_quant_append",
           "pikv_quant_attn_workspace_bytes", "pikv_quant_attn", "pikv_prompt_attn", "pikv_prompt_mass_workspace_bytes", "pikv_prompt_mass",
           "pikv_paged_fill", "pikv_paged_append", "pikv_paged_attn_workspace_bytes", "pikv_paged_attn")


class PikvError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, pikv_strerror(status), status))


class PikvDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("E", C.c_int32), ("S", C.c_int32), ("rank", C.c_int32), ("dtype", C.c_int32),
                ("stride_h", C.c_int64), ("stride_s", C.c_int64),
                ("route_rows_per_seq", C.c_int32), ("flags", C.c_int32), ("tq", C.c_int32),
                ("reserved", C.c_int32)]

    @property
    def width(self):
        return self.rank if self.rank else self.D


_lib = None
_native = None


def library_path() -> str:
    return _LIB_PATH


def is_built() -> bool:
    """Whether the library and the extension that makes its calls are there."""
    return os.path.exists(_LIB_PATH) and os.path.exists(_NATIVE_PATH)


def load_library():
    """dlopen libpikv.so (built by ``python -m paper_2508_06526_amd.build``).  Raises if absent."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise OSError("libpikv.so is not built: run `python -m paper_2508_06526_amd.build` "
                      "(there is no fallback path)")
    # The binding passes torch tensors and torch streams to the library, so both must talk to
    # ONE HIP runtime: torch brings its own copy of libamdhip64, and a libpikv.so opened before
    # torch would bind to the system's copy instead - its launches on torch's streams then fail
    # (PIKV_ERR_HIP).  Importing torch first makes the already-loaded runtime the one libpikv gets.
    import torch  # noqa: F401
    lib = C.CDLL(_LIB_PATH)
    vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
    dp = C.POINTER(PikvDesc)
    lib.pikv_route.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.pikv_route.restype = C.c_int
    lib.pikv_attn_workspace_bytes.argtypes = [dp, i32]
    lib.pikv_attn_workspace_bytes.restype = C.c_size_t
    lib.pikv_sharded_attn.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32,
                                      vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.pikv_sharded_attn.restype = C.c_int
    lib.pikv_sharded_attn_noalloc.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32,
                                              vp, vp, vp, vp, vp, vp]
    lib.pikv_sharded_attn_noalloc.restype = C.c_int
    lib.pikv_update_utility.argtypes = [dp, vp, vp, vp, vp, i32, f32, vp, vp]
    lib.pikv_update_utility.restype = C.c_int
    lib.pikv_policy_stamp.argtypes = [dp, vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp]
    lib.pikv_policy_stamp.restype = C.c_int
    lib.pikv_update_utility_tracked.argtypes = [dp, vp, vp, vp, vp, i32, f32, vp, f32, i32, vp, vp, vp]
    lib.pikv_update_utility_tracked.restype = C.c_int
    lib.pikv_policy_utility.argtypes = [dp, i32, vp, i32, f32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.pikv_policy_utility.restype = C.c_int
    lib.pikv_policy_compact.argtypes = [dp, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.pikv_policy_compact.restype = C.c_int
    lib.pikv_route_round_robin.argtypes = [i32, i32, i32, C.c_int64, vp, vp, vp]
    lib.pikv_route_round_robin.restype = C.c_int
    lib.pikv_evict.argtypes = [dp, vp, vp, i32, vp, i32, vp, vp, i32, i32, vp, vp, vp]
    lib.pikv_evict.restype = C.c_int
    lib.pikv_append.argtypes = [dp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.pikv_append.restype = C.c_int
    lib.pikv_strerror.argtypes = [C.c_int]
    lib.pikv_strerror.restype = C.c_char_p
    lib.pikv_decode_step.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, f32,
                                     vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.pikv_decode_step.restype = C.c_int
    lib.pikv_decode_step_policy.argtypes = list(lib.pikv_decode_step.argtypes) + [vp, vp]
    lib.pikv_decode_step_policy.restype = C.c_int
    lib.pikv_stream_read_probe.argtypes = [vp, i32, C.c_size_t, i32, vp, vp]
    lib.pikv_stream_read_probe.restype = C.c_int
    lib.pikv_router_penalty.argtypes = [i32, vp, i32, i32, i32, vp, vp, f32, vp, vp]
    lib.pikv_router_penalty.restype = C.c_int
    lib.pikv_compress.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp]
    lib.pikv_compress.restype = C.c_int
    lib.pikv_set_profile_events.argtypes = [vp, vp]
    lib.pikv_set_profile_events.restype = None
    lib.pikv_set_attn_split.argtypes = [i32]
    lib.pikv_set_attn_split.restype = None
    i64 = C.c_int64
    lib.pikv_norm_rope.argtypes = [vp, i32, i64, i32, i32, i32, i32, vp, vp, f32, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.pikv_norm_rope.restype = C.c_int
    lib.pikv_quant_pack.argtypes = [dp, i32, i32, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp]
    lib.pikv_quant_pack.restype = C.c_int
    lib.pikv_quant_read.argtypes = [dp, i32, i32, vp, vp, vp, vp, vp, vp, vp, i64, i64, vp]
    lib.pikv_quant_read.restype = C.c_int
    lib.pikv_quant_append.argtypes = [dp, i32, i32, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.pikv_quant_append.restype = C.c_int
    lib.pikv_quant_attn_workspace_bytes.argtypes = [dp, i32]
    lib.pikv_quant_attn_workspace_bytes.restype = C.c_size_t
    lib.pikv_quant_attn.argtypes = [dp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32,
                                    vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.pikv_quant_attn.restype = C.c_int
    lib.pikv_prompt_attn.argtypes = [vp, vp, vp, i32, i64, i64, i64, i32, i32, i32, i32, vp, i32, i32, vp, f32, f32, vp, i32, vp, vp, vp, vp]
    lib.pikv_prompt_attn.restype = C.c_int
    lib.pikv_prompt_mass_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.pikv_prompt_mass_workspace_bytes.restype = C.c_size_t
    lib.pikv_prompt_mass.argtypes = [vp, vp, i32, i64, i64, i32, i32, i32, i32, vp, i32, i32, vp, f32, f32, vp, i32, vp, vp, vp, vp,
                                     C.c_size_t, vp]
    lib.pikv_prompt_mass.restype = C.c_int
    pp = C.POINTER(PikvPages)
    lib.pikv_paged_fill.argtypes = [dp, pp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.pikv_paged_fill.restype = C.c_int
    lib.pikv_paged_append.argtypes = [dp, pp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.pikv_paged_append.restype = C.c_int
    lib.pikv_paged_attn_workspace_bytes.argtypes = [dp, i32]
    lib.pikv_paged_attn_workspace_bytes.restype = C.c_size_t
    lib.pikv_paged_attn.argtypes = [dp, pp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, f32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                    C.c_size_t, vp]
    lib.pikv_paged_attn.restype = C.c_int
    lib.pikv_version.argtypes = []
    lib.pikv_version.restype = C.c_int
    native = _load_native({name: C.cast(getattr(lib, name), C.c_void_p).value for name in EXPORTS})
    _lib, _native = lib, native
    return lib


class _NoExtension:
    """In place of an extension that is not there: leaves every call to the ctypes path."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_native(addresses):
    """The extension is tied to the Python and torch it was built against, libpikv.so to neither: without the extension the
    same kernels run, at 4 - 5 us more host time per call."""
    try:
        spec = importlib.util.spec_from_file_location("_pikv_native", _NATIVE_PATH)
        native = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(native)
    except (ImportError, OSError) as e:
        warnings.warn("calls go through ctypes: _pikv_native.so is not built for this Python and torch (%s); "
                      "run `python -m paper_2508_06526_amd.build`" % e, RuntimeWarning, stacklevel=3)
        return _NoExtension()
    native.setup(PikvDesc, PikvPolicyArgs, PikvRouterFeedback, PikvPages, addresses, _MARK)
    return native


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("storage dtype must be float32 or bfloat16, got %s" % t.dtype)


def _calls():
    """What makes the calls: the extension, or what stands in for it; loads the library if nothing has."""
    if _native is None:
        load_library()
    return _native


def _p(t):
    """Device address of a tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libpikv takes device memory only")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


_current_stream = None     # () -> hipStream_t of torch's current stream on the current device


def _stream(stream):
    global _current_stream
    if stream is not None:
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if _current_stream is None:
        import torch
        torch.cuda.current_stream()          # initialises the device
        try:
            raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
            _current_stream = lambda: raw(device())
        except AttributeError:
            _current_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _current_stream()


def _raw(stream):
    """A stream as the extension takes it: None (torch's current one) or an integer."""
    return None if stream is None else _stream(stream)


def _check(status, where):
    if status != 0:
        raise PikvError(status, where)


def make_desc(B, Hq, Hkv, D, E, S, rank=0, dtype=BF16, stride_h=None, stride_s=None,
              route_rows_per_seq=1, flags=0, tq=1) -> PikvDesc:
    w = rank if rank else D
    if stride_s is None:
        stride_s = w
    if stride_h is None:
        stride_h = S * stride_s
    return PikvDesc(B, Hq, Hkv, D, E, S, rank, dtype, stride_h, stride_s, route_rows_per_seq, flags, tq, 0)


def shard_table(shards, device=None):
    """Device array of B*E shard base addresses (entry b*E+e).

    ``shards`` is a tensor [B,E,Hkv,S,w] (one allocation) or a flat list of B*E tensors.  A table of int8 or float8_e4m3fn
    shards is marked as one: the calls on rows of the dense type, which would write behind such shards, refuse it (of
    shards of other types - raw bytes among them - nothing is known; PIKV_DESC_8BIT in the descriptor tells).
    """
    import torch
    if isinstance(shards, torch.Tensor):
        B, E = shards.shape[:2]
        step = shards.stride(1) * shards.element_size()
        assert shards.stride(0) == E * shards.stride(1)
        ptrs = [shards.data_ptr() + i * step for i in range(B * E)]
        device = shards.device
    else:
        ptrs = [s.data_ptr() for s in shards]
        device = shards[0].device
    table = torch.tensor(ptrs, dtype=torch.int64, device=device)
    if (shards if isinstance(shards, torch.Tensor) else shards[0]).dtype in (torch.int8, torch.float8_e4m3fn):
        setattr(table, _MARK, True)
    return table


_MARK = "_pikv_8bit"         # attribute of a table of 8-bit shards


def _dense(where, *tables):
    """Tables of shards of the dense type."""
    for t in tables:
        if getattr(t, _MARK, False):
            raise TypeError("%s: works on rows of the dense type, the table is of 8-bit shards" % where)


def pikv_strerror(status: int) -> str:
    return load_library().pikv_strerror(int(status)).decode()


def pikv_version() -> int:
    return load_library().pikv_version()


def pikv_set_attn_split(nsplit: int) -> None:
    load_library().pikv_set_attn_split(int(nsplit))


def pikv_set_profile_events(start, stop) -> None:
    """start/stop: torch.cuda.Event (timing enabled, already recorded once so that the HIP
    event exists) or None/None to switch the hook off."""
    h = lambda ev: None if ev is None else C.c_void_p(ev.cuda_event)
    load_library().pikv_set_profile_events(h(start), h(stop))


def pikv_route(x, W_r, bias, rows, d_r, E, k, topk_idx, gates, probs=None, stream=None):
    st = _calls().pikv_route(x, W_r, bias, rows, d_r, E, k, topk_idx, gates, probs, _raw(stream))
    if st is None:
        st = load_library().pikv_route(_p(x), _p(W_r), _p(bias), rows, d_r, E, k, _dtype_code(x),
                                       _p(topk_idx), _p(gates), _p(probs), _stream(stream))
    if st != 0:
        _check(st, "pikv_route")


def pikv_attn_workspace_bytes(desc: PikvDesc, k: int) -> int:
    return int(load_library().pikv_attn_workspace_bytes(C.byref(desc), k))


def pikv_sharded_attn(desc, q, K_shards, V_shards, U_K, U_V, n_valid, topk_idx, gates, k, combine,
                      scale, y, row_max, row_norm, scores, slot_coef, workspace, stream=None):
    st = _calls().pikv_sharded_attn(desc, q, K_shards, V_shards, U_K, U_V, n_valid, topk_idx, gates, k, combine, scale, y,
                                    row_max, row_norm, scores, slot_coef, workspace, _raw(stream))
    if st is None:
        _dense("pikv_sharded_attn", K_shards, V_shards)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        st = load_library().pikv_sharded_attn(
            C.byref(desc), _p(q), _p(K_shards), _p(V_shards), _p(U_K), _p(U_V), _p(n_valid),
            _p(topk_idx), _p(gates), k, combine, float(scale), _p(y), _p(row_max), _p(row_norm),
            _p(scores), _p(slot_coef), _p(workspace), ws_bytes, _stream(stream))
    if st != 0:
        _check(st, "pikv_sharded_attn")


NOALLOC_SCRATCH_BYTES = 4 << 20


def pikv_sharded_attn_noalloc(desc, q, K_shards, V_shards, U_K, U_V, n_valid, topk_idx, gates, k, combine,
                              scale, y, row_max, row_norm, scores, slot_coef, stream=None):
    st = _calls().pikv_sharded_attn_noalloc(desc, q, K_shards, V_shards, U_K, U_V, n_valid, topk_idx, gates, k, combine, scale,
                                            y, row_max, row_norm, scores, slot_coef, _raw(stream))
    if st is None:
        _dense("pikv_sharded_attn_noalloc", K_shards, V_shards)
        st = load_library().pikv_sharded_attn_noalloc(
            C.byref(desc), _p(q), _p(K_shards), _p(V_shards), _p(U_K), _p(U_V), _p(n_valid),
            _p(topk_idx), _p(gates), k, combine, float(scale), _p(y), _p(row_max), _p(row_norm),
            _p(scores), _p(slot_coef), _stream(stream))
    if st != 0:
        _check(st, "pikv_sharded_attn_noalloc")


def pikv_update_utility(desc, scores, slot_coef, n_valid, topk_idx, k, decay, utility, stream=None):
    st = _calls().pikv_update_utility(desc, scores, slot_coef, n_valid, topk_idx, k, decay, utility, _raw(stream))
    if st is None:
        st = load_library().pikv_update_utility(C.byref(desc), _p(scores), _p(slot_coef), _p(n_valid),
                                                _p(topk_idx), k, float(decay), _p(utility),
                                                _stream(stream))
    if st != 0:
        _check(st, "pikv_update_utility")


def pikv_evict(desc, utility, n_valid, capacity, sel_idx, sel_k, evicted_idx, evicted_cnt,
               max_evict, compact, K_shards, V_shards, stream=None):
    st = _calls().pikv_evict(desc, utility, n_valid, capacity, sel_idx, sel_k, evicted_idx, evicted_cnt, max_evict,
                             1 if compact else 0, K_shards, V_shards, _raw(stream))
    if st is None:
        if compact:
            _dense("pikv_evict", K_shards, V_shards)
        st = load_library().pikv_evict(C.byref(desc), _p(utility), _p(n_valid), capacity, _p(sel_idx),
                                       sel_k, _p(evicted_idx), _p(evicted_cnt), max_evict,
                                       1 if compact else 0, _p(K_shards), _p(V_shards), _stream(stream))
    if st != 0:
        _check(st, "pikv_evict")


def pikv_append(desc, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, K_shards,
                V_shards, utility, n_valid, stream=None):
    st = _calls().pikv_append(desc, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, K_shards, V_shards,
                              utility, n_valid, _raw(stream))
    if st is None:
        _dense("pikv_append", K_shards, V_shards)
        st = load_library().pikv_append(C.byref(desc), _p(K_new), _p(V_new), _p(topk_idx), k,
                                        _p(reuse_idx), _p(reuse_cnt), max_evict, _p(K_shards),
                                        _p(V_shards), _p(utility), _p(n_valid), _stream(stream))
    if st != 0:
        _check(st, "pikv_append")


def pikv_decode_step(desc, q, W_r, bias, K_new, V_new, K_shards, V_shards, U_K, U_V, n_valid, utility,
                     k, combine, scale, decay, topk_idx, gates, evicted_idx, evicted_cnt, y, row_max,
                     row_norm, scores, slot_coef, workspace, stream=None):
    st = _calls().pikv_decode_step(desc, q, W_r, bias, K_new, V_new, K_shards, V_shards, U_K, U_V, n_valid, utility, k,
                                   combine, scale, decay, topk_idx, gates, evicted_idx, evicted_cnt, y, row_max,
                                   row_norm, scores, slot_coef, workspace, _raw(stream))
    if st is None:
        _dense("pikv_decode_step", K_shards, V_shards)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        st = load_library().pikv_decode_step(
            C.byref(desc), _p(q), _p(W_r), _p(bias), _p(K_new), _p(V_new), _p(K_shards), _p(V_shards),
            _p(U_K), _p(U_V), _p(n_valid), _p(utility), k, combine, float(scale), float(decay),
            _p(topk_idx), _p(gates), _p(evicted_idx), _p(evicted_cnt), _p(y), _p(row_max), _p(row_norm),
            _p(scores), _p(slot_coef), _p(workspace), ws_bytes, _stream(stream))
    if st != 0:
        _check(st, "pikv_decode_step")


def pikv_stream_read_probe(bufs, n, bytes_each, parts, out, stream=None):
    st = load_library().pikv_stream_read_probe(_p(bufs), n, bytes_each, parts, _p(out), _stream(stream))
    _check(st, "pikv_stream_read_probe")


def pikv_router_penalty(mode, topk_idx, rows, k, E, load, miss, coef, bias, stream=None):
    st = _calls().pikv_router_penalty(mode, topk_idx, rows, k, E, load, miss, coef, bias, _raw(stream))
    if st is None:
        st = load_library().pikv_router_penalty(mode, _p(topk_idx), rows, k, E, _p(load), _p(miss),
                                                float(coef), _p(bias), _stream(stream))
    if st != 0:
        _check(st, "pikv_router_penalty")


def pikv_compress(desc, K_full, Wenc_K, K_codes, V_full=None, Wenc_V=None, V_codes=None, stream=None):
    st = _calls().pikv_compress(desc, K_full, Wenc_K, K_codes, V_full, Wenc_V, V_codes, _raw(stream))
    if st is None:
        st = load_library().pikv_compress(C.byref(desc), _p(K_full), _p(Wenc_K), _p(K_codes), _p(V_full),
                                          _p(Wenc_V), _p(V_codes), _stream(stream))
    if st != 0:
        _check(st, "pikv_compress")


def pikv_policy_stamp(desc, topk_idx, k, reuse_idx, reuse_cnt, max_evict, n_valid, now, birth,
                      last_access, freq, stream=None):
    st = _calls().pikv_policy_stamp(desc, topk_idx, k, reuse_idx, reuse_cnt, max_evict, n_valid, now, birth,
                                    last_access, freq, _raw(stream))
    if st is None:
        st = load_library().pikv_policy_stamp(C.byref(desc), _p(topk_idx), k, _p(reuse_idx), _p(reuse_cnt),
                                              max_evict, _p(n_valid), int(now), _p(birth), _p(last_access),
                                              _p(freq), _stream(stream))
    if st != 0:
        _check(st, "pikv_policy_stamp")


def pikv_update_utility_tracked(desc, scores, slot_coef, n_valid, topk_idx, k, decay, utility, threshold,
                                now, last_access, freq, stream=None):
    st = _calls().pikv_update_utility_tracked(desc, scores, slot_coef, n_valid, topk_idx, k, decay, utility, threshold,
                                              now, last_access, freq, _raw(stream))
    if st is None:
        st = load_library().pikv_update_utility_tracked(C.byref(desc), _p(scores), _p(slot_coef), _p(n_valid),
                                                        _p(topk_idx), k, float(decay), _p(utility),
                                                        float(threshold), int(now), _p(last_access), _p(freq),
                                                        _stream(stream))
    if st != 0:
        _check(st, "pikv_update_utility_tracked")


def pikv_policy_utility(desc, policy, n_valid, now, lam, window, protect, birth, last_access, freq, h2o,
                        out, stream=None):
    st = _calls().pikv_policy_utility(desc, policy, n_valid, now, lam, window, protect, birth, last_access, freq, h2o, out, _raw(stream))
    if st is None:
        st = load_library().pikv_policy_utility(C.byref(desc), int(policy), _p(n_valid), int(now), float(lam),
                                                int(window), int(protect), _p(birth), _p(last_access),
                                                _p(freq), _p(h2o), _p(out), _stream(stream))
    if st != 0:
        _check(st, "pikv_policy_utility")


def pikv_policy_compact(desc, evicted_idx, evicted_cnt, max_evict, n_valid, birth, last_access, freq,
                        stream=None):
    st = _calls().pikv_policy_compact(desc, evicted_idx, evicted_cnt, max_evict, n_valid, birth, last_access, freq, _raw(stream))
    if st is None:
        st = load_library().pikv_policy_compact(C.byref(desc), _p(evicted_idx), _p(evicted_cnt), max_evict,
                                                _p(n_valid), _p(birth), _p(last_access), _p(freq), _stream(stream))
    if st != 0:
        _check(st, "pikv_policy_compact")


class PikvPolicyArgs(C.Structure):
    _fields_ = [("policy", C.c_int32), ("now", C.c_int32), ("lam", C.c_float), ("window", C.c_int32),
                ("protect", C.c_int32), ("threshold", C.c_float), ("birth", C.c_void_p),
                ("last_access", C.c_void_p), ("freq", C.c_void_p)]


def make_policy_args(policy, now, lam=0.0, window=0, protect=0, threshold=0.0, birth=None, last_access=None,
                     freq=None):
    return PikvPolicyArgs(int(policy), int(now), float(lam), int(window), int(protect), float(threshold), _p(birth),
                          _p(last_access), _p(freq))


class PikvRouterFeedback(C.Structure):
    _fields_ = [("mode", C.c_int32), ("coef", C.c_float), ("load", C.c_void_p), ("miss", C.c_void_p),
                ("bias", C.c_void_p)]


def make_router_feedback(mode, coef, load, bias, miss=None):
    return PikvRouterFeedback(int(mode), float(coef), _p(load), _p(miss), _p(bias))


def pikv_decode_step_policy(desc, q, W_r, bias, K_new, V_new, K_shards, V_shards, U_K, U_V, n_valid, utility, k,
                            combine, scale, decay, topk_idx, gates, evicted_idx, evicted_cnt, y, row_max,
                            row_norm, scores, slot_coef, workspace, policy_args, feedback=None, stream=None):
    st = _calls().pikv_decode_step_policy(desc, q, W_r, bias, K_new, V_new, K_shards, V_shards, U_K, U_V, n_valid, utility, k,
                                          combine, scale, decay, topk_idx, gates, evicted_idx, evicted_cnt, y, row_max,
                                          row_norm, scores, slot_coef, workspace, _raw(stream), policy_args, feedback)
    if st is None:
        _dense("pikv_decode_step_policy", K_shards, V_shards)
        st = load_library().pikv_decode_step_policy(
            C.byref(desc), _p(q), _p(W_r), _p(bias), _p(K_new), _p(V_new), _p(K_shards), _p(V_shards), _p(U_K),
            _p(U_V), _p(n_valid), _p(utility), k, combine, float(scale), float(decay), _p(topk_idx), _p(gates),
            _p(evicted_idx), _p(evicted_cnt), _p(y), _p(row_max), _p(row_norm), _p(scores), _p(slot_coef),
            _p(workspace), workspace.numel() * workspace.element_size(), _stream(stream),
            None if policy_args is None else C.cast(C.pointer(policy_args), C.c_void_p),
            None if feedback is None else C.cast(C.pointer(feedback), C.c_void_p))
    if st != 0:
        _check(st, "pikv_decode_step_policy")


def pikv_route_round_robin(rows, E, k, step, topk_idx, gates, stream=None):
    st = load_library().pikv_route_round_robin(rows, E, k, int(step), _p(topk_idx), _p(gates), _stream(stream))
    _check(st, "pikv_route_round_robin")


# ---- Operators around an 8-bit cache.  What these pass on is checked here as well: the type of every tensor, that all are
# on one device, whose current stream they then use and which is current during the call, and that each holds what the
# call reads or writes of it.
def _typed(where, want, *tensors):
    for t in tensors:
        if t is not None and t.dtype != want:
            raise TypeError("%s: expected a tensor of %s, got %s" % (where, want, t.dtype))


def _storage(desc):
    import torch
    return torch.float32 if desc.dtype == F32 else torch.bfloat16


def _on_device(where, call, stream, tensors):
    """call(stream handle) with the tensors' device current.  ``tensors``: (name, tensor, the elements it must hold at least[, the
    last dimension it must have if it has four])."""
    import torch
    device = None
    for _, t, *_ in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("libpikv takes device memory only")
        if device is not None and t.device != device:
            raise ValueError("%s: tensors on %s and %s" % (where, device, t.device))
        device = t.device
    if device is None:
        raise ValueError("%s: no tensor given" % where)
    _holds(where, tensors)
    with torch.cuda.device(device):
        return call(_stream(stream))


def _holds(where, tensors):
    for name, t, least, *last in tensors:
        if t is None:
            continue
        if t.numel() < least:
            raise ValueError("%s: %s has %d elements, %d are needed" % (where, name, t.numel(), least))
        if last and t.dim() == 4 and t.numel() > 0 and t.shape[-1] != last[0]:
            raise ValueError("%s: the last dimension of %s is %d, not %d" % (where, name, t.shape[-1], last[0]))


def _int32_float32(where, integers, floats, tables=()):
    import torch
    _typed(where, torch.int32, *integers)
    _typed(where, torch.float32, *floats)
    _typed(where, torch.int64, *tables)          # of shard addresses, not the shards


def _rows(x, token_stride):
    """Device address of rows that need not be contiguous: a slice of a wider projection."""
    if (x.stride(-1) != 1 and x.shape[-1] > 1) or (x.dim() > 2 and x.shape[1] > 1 and x.stride(1) != x.shape[2]):
        raise ValueError("the values of a row must be contiguous")
    if x.dim() > 1 and not x.is_contiguous() and x.stride(0) != token_stride:
        raise ValueError("rows are %d elements apart, token_stride is %d" % (x.stride(0), token_stride))
    return x.data_ptr()


def _rope_tensors(x, tokens, token_stride, Hq, Hkv, D, w_q, w_k, positions, inv_freq, rotary_dim, q_out, k_out, v_out):
    row = (Hq + Hkv * (1 if v_out is None else 2)) * D
    if x.is_contiguous():
        rows = ("x", x, (tokens - 1) * token_stride + row if tokens > 0 else 0)
    else:                                        # rows token_stride apart, each with what the view has of it
        rows = ("x", x, max(tokens * x[:1].numel(), x.shape[0] * row if tokens > 0 else 0))
    rotated = rotary_dim > 0
    return [rows, ("w_q", w_q, D), ("w_k", w_k, D), ("positions", positions, tokens if rotated else 0),
            ("inv_freq", inv_freq, rotary_dim // 2), ("q_out", q_out, tokens * Hq * D), ("k_out", k_out, tokens * Hkv * D),
            ("v_out", v_out, tokens * Hkv * D)]


def _cache_tensors(desc, block, K_shards, V_shards, K_scales, V_scales, n_valid):
    be = desc.B * desc.E
    blocks = (desc.S - 1) // block + 1 if block > 0 else 0
    return [("K_shards", K_shards, be), ("V_shards", V_shards, be), ("K_scales", K_scales, be * desc.Hkv * blocks, blocks),
            ("V_scales", V_scales, be * desc.Hkv * blocks, blocks), ("n_valid", n_valid, be)]


def _append_tensors(desc, block, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, K_shards, V_shards, K_scales, V_scales,
                    utility, n_valid):
    be, row = desc.B * desc.E, desc.B * desc.Hkv * desc.D
    return _cache_tensors(desc, block, K_shards, V_shards, K_scales, V_scales, n_valid) + [
        ("K_new", K_new, row), ("V_new", V_new, row), ("topk_idx", topk_idx, desc.B * k), ("reuse_idx", reuse_idx, be * max_evict),
        ("reuse_cnt", reuse_cnt, be), ("utility", utility, be * desc.S)]


def _attn_tensors(desc, block, q, K_shards, V_shards, K_scales, V_scales, n_valid, topk_idx, gates, k, y, row_max, row_norm, scores,
                  slot_coef, workspace):
    heads = desc.B * desc.Hq
    selected = desc.B * desc.route_rows_per_seq * k
    return _cache_tensors(desc, block, K_shards, V_shards, K_scales, V_scales, n_valid) + [
        ("q", q, heads * desc.D), ("topk_idx", topk_idx, selected), ("gates", gates, selected), ("y", y, heads * desc.D),
        ("row_max", row_max, heads), ("row_norm", row_norm, heads), ("scores", scores, heads * k * desc.S, desc.S),
        ("slot_coef", slot_coef, heads * k * 2), ("workspace", workspace, 0)]


def pikv_norm_rope(x, tokens, token_stride, Hq, Hkv, D, w_q, w_k, eps, positions, inv_freq, rotary_dim, interleaved, q_out,
                   k_out, v_out=None, stream=None):
    """``x``: [tokens, heads * D] or [tokens, heads, D], rows ``token_stride`` elements apart (a view into a wider projection is
    taken as it is)."""
    where = "pikv_norm_rope"
    st = _calls().pikv_norm_rope(x, tokens, token_stride, Hq, Hkv, D, w_q, w_k, eps, positions, inv_freq, rotary_dim,
                                 1 if interleaved else 0, q_out, k_out, v_out, _raw(stream))
    if st is None:
        _typed(where, x.dtype, w_q, w_k, q_out, k_out, v_out)
        _int32_float32(where, [positions], [inv_freq])
        st = _on_device(where, lambda s: load_library().pikv_norm_rope(
            _rows(x, token_stride), tokens, token_stride, Hq, Hkv, D, _dtype_code(x), _p(w_q), _p(w_k), float(eps), _p(positions),
            _p(inv_freq), rotary_dim, 1 if interleaved else 0, _p(q_out), _p(k_out), _p(v_out), s),
            stream, _rope_tensors(x, tokens, token_stride, Hq, Hkv, D, w_q, w_k, positions, inv_freq, rotary_dim, q_out, k_out, v_out))
    if st != 0:
        _check(st, where)


def pikv_quant_pack(desc, format, block, K_dense, V_dense, dense_stride_h, dense_stride_s, n_valid, K_shards, V_shards, K_scales,
                    V_scales, stream=None):
    where = "pikv_quant_pack"
    st = _calls().pikv_quant_pack(desc, format, block, K_dense, V_dense, dense_stride_h, dense_stride_s, n_valid, K_shards, V_shards,
                                  K_scales, V_scales, _raw(stream))
    if st is None:
        _dense(where, K_dense, V_dense)
        _int32_float32(where, [n_valid], [K_scales, V_scales], [K_dense, V_dense, K_shards, V_shards])
        st = _on_device(where, lambda s: load_library().pikv_quant_pack(
            C.byref(desc), format, block, _p(K_dense), _p(V_dense), dense_stride_h, dense_stride_s, _p(n_valid), _p(K_shards),
            _p(V_shards), _p(K_scales), _p(V_scales), s), stream,
            _cache_tensors(desc, block, K_shards, V_shards, K_scales, V_scales, n_valid) + [
                ("K_dense", K_dense, desc.B * desc.E), ("V_dense", V_dense, desc.B * desc.E)])
    if st != 0:
        _check(st, where)


def pikv_quant_read(desc, format, block, K_shards, V_shards, K_scales, V_scales, n_valid, K_dense, V_dense, dense_stride_h,
                    dense_stride_s, stream=None):
    where = "pikv_quant_read"
    st = _calls().pikv_quant_read(desc, format, block, K_shards, V_shards, K_scales, V_scales, n_valid, K_dense, V_dense,
                                  dense_stride_h, dense_stride_s, _raw(stream))
    if st is None:
        _dense(where, K_dense, V_dense)
        _int32_float32(where, [n_valid], [K_scales, V_scales], [K_dense, V_dense, K_shards, V_shards])
        st = _on_device(where, lambda s: load_library().pikv_quant_read(
            C.byref(desc), format, block, _p(K_shards), _p(V_shards), _p(K_scales), _p(V_scales), _p(n_valid), _p(K_dense),
            _p(V_dense), dense_stride_h, dense_stride_s, s), stream,
            _cache_tensors(desc, block, K_shards, V_shards, K_scales, V_scales, n_valid) + [
                ("K_dense", K_dense, desc.B * desc.E), ("V_dense", V_dense, desc.B * desc.E)])
    if st != 0:
        _check(st, where)


def pikv_quant_append(desc, format, block, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, K_shards, V_shards, K_scales,
                      V_scales, utility, n_valid, stream=None):
    where = "pikv_quant_append"
    st = _calls().pikv_quant_append(desc, format, block, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, K_shards,
                                    V_shards, K_scales, V_scales, utility, n_valid, _raw(stream))
    if st is None:
        _typed(where, _storage(desc), K_new, V_new)
        _int32_float32(where, [topk_idx, reuse_idx, reuse_cnt, n_valid], [K_scales, V_scales, utility], [K_shards, V_shards])
        st = _on_device(where, lambda s: load_library().pikv_quant_append(
            C.byref(desc), format, block, _p(K_new), _p(V_new), _p(topk_idx), k, _p(reuse_idx), _p(reuse_cnt), max_evict,
            _p(K_shards), _p(V_shards), _p(K_scales), _p(V_scales), _p(utility), _p(n_valid), s), stream,
            _append_tensors(desc, block, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, K_shards, V_shards, K_scales,
                            V_scales, utility, n_valid))
    if st != 0:
        _check(st, where)


def pikv_quant_attn_workspace_bytes(desc: PikvDesc, k: int) -> int:
    return int(load_library().pikv_quant_attn_workspace_bytes(C.byref(desc), k))


def pikv_quant_attn(desc, format, block, q, K_shards, V_shards, K_scales, V_scales, n_valid, topk_idx, gates, k, combine, scale, y,
                    row_max, row_norm, scores, slot_coef, workspace, stream=None):
    where = "pikv_quant_attn"
    st = _calls().pikv_quant_attn(desc, format, block, q, K_shards, V_shards, K_scales, V_scales, n_valid, topk_idx, gates, k, combine,
                                  scale, y, row_max, row_norm, scores, slot_coef, workspace, _raw(stream))
    if st is None:
        _typed(where, _storage(desc), q)
        _int32_float32(where, [n_valid, topk_idx], [K_scales, V_scales, gates, y, row_max, row_norm, scores, slot_coef],
                       [K_shards, V_shards])
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        st = _on_device(where, lambda s: load_library().pikv_quant_attn(
            C.byref(desc), format, block, _p(q), _p(K_shards), _p(V_shards), _p(K_scales), _p(V_scales), _p(n_valid), _p(topk_idx),
            _p(gates), k, combine, float(scale), _p(y), _p(row_max), _p(row_norm), _p(scores), _p(slot_coef), _p(workspace), ws_bytes,
            s), stream, _attn_tensors(desc, block, q, K_shards, V_shards, K_scales, V_scales, n_valid, topk_idx, gates, k, y, row_max,
                                      row_norm, scores, slot_coef, workspace))
    if st != 0:
        _check(st, where)


# ---- Between a prompt and a paged cache (checked as the calls above).
class PikvPages(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page", C.c_int32), ("stride_page", C.c_int64), ("stride_h", C.c_int64), ("stride_s", C.c_int64)]


def make_pages(n_pages, page, Hkv, D, stride_page=None, stride_h=None, stride_s=None) -> PikvPages:
    """Geometry of pools [n_pages, Hkv, page, D], or with strides (elements) of others: a pool of one tensor [n_pages, 2, Hkv, page, D]
    for K and V has stride_page = 2 * Hkv * page * D, pages [n_pages, page, Hkv, D] have stride_h = D, stride_s = Hkv * D."""
    if stride_s is None:
        stride_s = D
    if stride_h is None:
        stride_h = page * stride_s
    if stride_page is None:
        stride_page = max(Hkv * stride_h, page * stride_s)
    return PikvPages(n_pages, page, stride_page, stride_h, stride_s)


def _pool(where, pool, desc, pages):
    """Device address of a pool, which may be a part of a larger tensor: what lies behind it has to hold the pages."""
    if pool is None:
        return None
    if not pool.is_cuda:
        raise ValueError("libpikv takes device memory only")
    extent = (pages.n_pages - 1) * pages.stride_page + (desc.Hkv - 1) * pages.stride_h + (pages.page - 1) * pages.stride_s + desc.D
    held = pool.untyped_storage().nbytes() // pool.element_size() - pool.storage_offset()
    if pool.is_contiguous():
        held = min(held, pool.numel())
    if desc.B > 0 and held < extent:
        raise ValueError("%s: a pool holds %d elements, its pages take %d" % (where, held, extent))
    if pool.dim() > 0 and pool.shape[-1] > 1 and pool.stride(-1) != 1:
        raise ValueError("the values of a row must be contiguous")
    return pool.data_ptr()


def _paged_tensors(desc, pages, page_table, n_valid, entry_pos):
    be = desc.B * desc.E
    per_shard = (desc.S - 1) // pages.page + 1 if pages.page > 0 else 0
    return [("page_table", page_table, be * per_shard), ("n_valid", n_valid, be), ("entry_pos", entry_pos, be * desc.S)]


def _prompt_tensors(q, k, v, tokens, q_stride, k_stride, v_stride, Hq, Hkv, D, cu_seqlens, B, prefix, slopes, row_max, row_norm):
    def rows(name, x, stride, heads):
        if x is None:
            return (name, x, 0)
        if x.is_contiguous():
            return (name, x, (tokens - 1) * stride + heads * D if tokens > 0 else 0)
        return (name, x, max(tokens * x[:1].numel(), x.shape[0] * heads * D if tokens > 0 else 0))
    return [rows("q", q, q_stride, Hq), rows("k", k, k_stride, Hkv), rows("v", v, v_stride, Hkv), ("cu_seqlens", cu_seqlens, B + 1),
            ("prefix", prefix, B), ("slopes", slopes, Hq), ("row_max", row_max, tokens * Hq), ("row_norm", row_norm, tokens * Hq)]


def pikv_prompt_attn(q, k, v, tokens, q_stride, k_stride, v_stride, Hq, Hkv, D, cu_seqlens, B, max_len, prefix, scale, cap, slopes, window,
                     out, row_max=None, row_norm=None, stream=None):
    """``q``, ``k``, ``v``: [tokens, heads * D] or [tokens, heads, D], rows ``*_stride`` elements apart (views into a wider projection are
    taken as they are)."""
    where = "pikv_prompt_attn"
    st = _calls().pikv_prompt_attn(q, k, v, tokens, q_stride, k_stride, v_stride, Hq, Hkv, D, cu_seqlens, B, max_len, prefix, scale, cap,
                                   slopes, window, out, row_max, row_norm, _raw(stream))
    if st is None:
        _typed(where, q.dtype, k, v, out)
        _int32_float32(where, [cu_seqlens, prefix], [slopes, row_max, row_norm])
        st = _on_device(where, lambda s: load_library().pikv_prompt_attn(
            _rows(q, q_stride), _rows(k, k_stride), _rows(v, v_stride), tokens, q_stride, k_stride, v_stride, Hq, Hkv, D, _dtype_code(q),
            _p(cu_seqlens), B, max_len, _p(prefix), float(scale), float(cap), _p(slopes), window, _p(out), _p(row_max), _p(row_norm), s),
            stream, _prompt_tensors(q, k, v, tokens, q_stride, k_stride, v_stride, Hq, Hkv, D, cu_seqlens, B, prefix, slopes, row_max,
                                    row_norm) + [("out", out, tokens * Hq * D)])
    if st != 0:
        _check(st, where)


def pikv_prompt_mass_workspace_bytes(tokens, Hkv, B, max_len) -> int:
    return int(load_library().pikv_prompt_mass_workspace_bytes(tokens, Hkv, B, max_len))


def pikv_prompt_mass(q, k, tokens, q_stride, k_stride, Hq, Hkv, D, cu_seqlens, B, max_len, prefix, scale, cap, slopes, window, row_max,
                     row_norm, mass, workspace, stream=None):
    where = "pikv_prompt_mass"
    st = _calls().pikv_prompt_mass(q, k, tokens, q_stride, k_stride, Hq, Hkv, D, cu_seqlens, B, max_len, prefix, scale, cap, slopes, window,
                                   row_max, row_norm, mass, workspace, _raw(stream))
    if st is None:
        _typed(where, q.dtype, k)
        _int32_float32(where, [cu_seqlens, prefix], [slopes, row_max, row_norm, mass])
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        st = _on_device(where, lambda s: load_library().pikv_prompt_mass(
            _rows(q, q_stride), _rows(k, k_stride), tokens, q_stride, k_stride, Hq, Hkv, D, _dtype_code(q), _p(cu_seqlens), B, max_len,
            _p(prefix), float(scale), float(cap), _p(slopes), window, _p(row_max), _p(row_norm), _p(mass), _p(workspace), ws_bytes, s),
            stream, _prompt_tensors(q, k, None, tokens, q_stride, k_stride, 0, Hq, Hkv, D, cu_seqlens, B, prefix, slopes, row_max,
                                    row_norm) + [("mass", mass, tokens), ("workspace", workspace, 0)])
    if st != 0:
        _check(st, where)


def pikv_paged_fill(desc, pages, K_new, V_new, tokens, cu_seqlens, topk_idx, k, weight, positions, K_pool, V_pool, page_table, entry_pos,
                    utility, n_valid, slots, stream=None):
    where = "pikv_paged_fill"
    st = _calls().pikv_paged_fill(desc, pages, K_new, V_new, tokens, cu_seqlens, topk_idx, k, weight, positions, K_pool, V_pool, page_table,
                                  entry_pos, utility, n_valid, slots, _raw(stream))
    if st is None:
        _typed(where, _storage(desc), K_new, V_new, K_pool, V_pool)
        _int32_float32(where, [cu_seqlens, topk_idx, positions, page_table, entry_pos, n_valid, slots], [weight, utility])
        row = desc.Hkv * desc.D
        st = _on_device(where, lambda s: load_library().pikv_paged_fill(
            C.byref(desc), C.byref(pages), _p(K_new), _p(V_new), tokens, _p(cu_seqlens), _p(topk_idx), k, _p(weight), _p(positions),
            _pool(where, K_pool, desc, pages), _pool(where, V_pool, desc, pages), _p(page_table), _p(entry_pos), _p(utility), _p(n_valid),
            _p(slots), s), stream, _paged_tensors(desc, pages, page_table, n_valid, entry_pos) + [
                ("K_new", K_new, tokens * row), ("V_new", V_new, tokens * row), ("cu_seqlens", cu_seqlens, desc.B + 1),
                ("topk_idx", topk_idx, tokens * k), ("weight", weight, tokens), ("positions", positions, tokens), ("K_pool", K_pool, 0),
                ("V_pool", V_pool, 0), ("utility", utility, desc.B * desc.E * desc.S), ("slots", slots, tokens * k)])
    if st != 0:
        _check(st, where)


def pikv_paged_append(desc, pages, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, positions, K_pool, V_pool, page_table, entry_pos,
                      utility, n_valid, stream=None):
    where = "pikv_paged_append"
    st = _calls().pikv_paged_append(desc, pages, K_new, V_new, topk_idx, k, reuse_idx, reuse_cnt, max_evict, positions, K_pool, V_pool,
                                    page_table, entry_pos, utility, n_valid, _raw(stream))
    if st is None:
        _typed(where, _storage(desc), K_new, V_new, K_pool, V_pool)
        _int32_float32(where, [topk_idx, reuse_idx, reuse_cnt, positions, page_table, entry_pos, n_valid], [utility])
        row, be = desc.B * desc.Hkv * desc.D, desc.B * desc.E
        st = _on_device(where, lambda s: load_library().pikv_paged_append(
            C.byref(desc), C.byref(pages), _p(K_new), _p(V_new), _p(topk_idx), k, _p(reuse_idx), _p(reuse_cnt), max_evict, _p(positions),
            _pool(where, K_pool, desc, pages), _pool(where, V_pool, desc, pages), _p(page_table), _p(entry_pos), _p(utility), _p(n_valid), s),
            stream, _paged_tensors(desc, pages, page_table, n_valid, entry_pos) + [
                ("K_new", K_new, row), ("V_new", V_new, row), ("topk_idx", topk_idx, desc.B * k), ("reuse_idx", reuse_idx, be * max_evict),
                ("reuse_cnt", reuse_cnt, be), ("positions", positions, desc.B), ("K_pool", K_pool, 0), ("V_pool", V_pool, 0),
                ("utility", utility, be * desc.S)])
    if st != 0:
        _check(st, where)


def pikv_paged_attn_workspace_bytes(desc: PikvDesc, k: int) -> int:
    return int(load_library().pikv_paged_attn_workspace_bytes(C.byref(desc), k))


def pikv_paged_attn(desc, pages, q, K_pool, V_pool, page_table, n_valid, topk_idx, gates, k, combine, scale, cap, slopes, window, prefix,
                    entry_pos, q_pos, y, row_max, row_norm, scores, slot_coef, workspace, stream=None):
    where = "pikv_paged_attn"
    st = _calls().pikv_paged_attn(desc, pages, q, K_pool, V_pool, page_table, n_valid, topk_idx, gates, k, combine, scale, cap, slopes, window,
                                  prefix, entry_pos, q_pos, y, row_max, row_norm, scores, slot_coef, workspace, _raw(stream))
    if st is None:
        _typed(where, _storage(desc), q, K_pool, V_pool)
        _int32_float32(where, [page_table, n_valid, topk_idx, prefix, entry_pos, q_pos], [gates, slopes, y, row_max, row_norm, scores, slot_coef])
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        heads, tq = desc.B * desc.Hq, max(desc.tq, 1)
        selected = desc.B * desc.route_rows_per_seq * k
        st = _on_device(where, lambda s: load_library().pikv_paged_attn(
            C.byref(desc), C.byref(pages), _p(q), _pool(where, K_pool, desc, pages), _pool(where, V_pool, desc, pages), _p(page_table),
            _p(n_valid), _p(topk_idx), _p(gates), k, combine, float(scale), float(cap), _p(slopes), window, _p(prefix), _p(entry_pos), _p(q_pos),
            _p(y), _p(row_max), _p(row_norm), _p(scores), _p(slot_coef), _p(workspace), ws_bytes, s), stream,
            _paged_tensors(desc, pages, page_table, n_valid, entry_pos) + [
                ("q", q, heads * desc.D), ("K_pool", K_pool, 0), ("V_pool", V_pool, 0), ("topk_idx", topk_idx, selected), ("gates", gates, selected),
                ("slopes", slopes, desc.Hq // tq), ("prefix", prefix, desc.B), ("q_pos", q_pos, desc.B * tq), ("y", y, heads * desc.D),
                ("row_max", row_max, heads), ("row_norm", row_norm, heads), ("scores", scores, heads * k * desc.S, desc.S),
                ("slot_coef", slot_coef, heads * k * 2), ("workspace", workspace, 0)])
    if st != 0:
        _check(st, where)
