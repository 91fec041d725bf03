"""ctypes binding of libexpertweave.so: argument marshalling only.

Every step of the hot path runs inside the library's HIP kernels; PyTorch supplies device
memory and the current stream.  There is no fallback: if the library is missing or a call
fails, an exception is raised.  Function names mirror include/expertweave.h.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libexpertweave.so")

EW_F32, EW_BF16 = 0, 1
EW_POOL_VMM, EW_POOL_PADDED, EW_POOL_FAKE, EW_POOL_EAGER_UNMAP = 0, 1, 2, 4
ERR_NAMES = {0: "EW_OK", -1: "EW_ERR_INVALID_ARG", -2: "EW_ERR_OOM", -3: "EW_ERR_VMM", -4: "EW_ERR_STATE",
             -5: "EW_ERR_WORKSPACE", -6: "EW_ERR_UNSUPPORTED", -7: "EW_ERR_HIP"}

# name -> (restype, argtypes); mirrors include/expertweave.h
_i32p, _f32p, _vp, _sz, _int = C.POINTER(C.c_int32), C.POINTER(C.c_float), C.c_void_p, C.c_size_t, C.c_int
SIGNATURES = {
    "ew_last_error": (C.c_char_p, []),
    "ew_abi_version": (_int, []),
    "expert_pool_create": (_int, [C.POINTER(_vp), _int, _int, _int, _int, _int, _sz, _sz, _sz, _sz, _int]),
    "expert_pool_destroy": (_int, [_vp]),
    "expert_pool_map": (_int, [_vp, _int, _int, _int, _vp, _vp, _vp, _vp]),
    "expert_pool_unmap": (_int, [_vp, _int, _int, _vp]),
    "expert_pool_view": (_int, [_vp, _int, C.POINTER(_vp), C.POINTER(_vp), C.POINTER(_vp), C.POINTER(_int)]),
    "expert_pool_expert_map_host": (_int, [_vp, _int, _vp]),
    "expert_pool_touch": (_int, [_vp, _int, _vp]),
    "expert_pool_lru_victim": (_int, [_vp, C.POINTER(C.c_int)]),
    "expert_pool_stats": (_int, [_vp, _vp]),
    "expert_pool_trim": (_int, [_vp, _sz]),
    "expert_pool_fake_fail_at": (_int, [_vp, _int, _int]),
    "expert_pool_fake_is_mapped": (_int, [_vp, _int, _int, _sz, C.POINTER(_int)]),
    "moe_route_topk": (_int, [_vp, _int, _int, _int, _int, _vp, _vp, _vp]),
    "moe_reroute_permute_workspace_bytes": (_sz, [_int, _int, _int]),
    "moe_reroute_permute": (_int, [_vp, _vp, _vp, _int, _int, _int, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "moe_reroute_permute_static_max_bytes": (_sz, []),
    "moe_reroute_permute_static": (_int, [_vp, _vp, _vp, _int, _int, _int, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp]),
    "moe_route_reroute_permute": (_int, [_vp, _vp, _vp, _int, _int, _int, _int, _int, _int, _vp, _vp, _vp, _vp, _vp,
                                         _vp, _vp, _vp, _sz, _vp]),
    "moe_route_reroute_permute_plan": (_int, [_vp, _vp, _vp, _int, _int, _int, _int, _int, _int, _vp, _vp, _vp, _vp, _vp,
                                              _vp, _vp, _vp, _sz, _int, _int, _int, _int, _vp, _sz, _vp]),
    "moe_reroute_singleop_workspace_bytes": (_sz, [_int, _int]),
    "moe_reroute_singleop": (_int, [_vp, _vp, _vp, _int, _int, _int, _int, _vp, _vp, _sz, _vp]),
    "moe_grouped_ffn_workspace_bytes": (_sz, [_int, _int, _int, _int, _int, _int]),
    "moe_grouped_ffn": (_int, [_vp, _int, _int, _int, _int, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "moe_grouped_ffn_planned": (_int, [_vp, _int, _int, _int, _int, _int, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                       _vp, _vp, _sz, _vp]),
    "moe_grouped_ffn_with_shared": (_int, [_vp, _int, _int, _int, _int, _int, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                           _vp, _vp, _sz, _vp]),
    "moe_unpermute": (_int, [_vp, _vp, _vp, _vp, _int, _vp, _int, _int, _int, _int, _vp, _vp]),
    "moe_unpermute_rmsnorm": (_int, [_vp, _vp, _vp, _vp, _int, _vp, _int, _int, _int, _int, _vp, C.c_float, _vp, _vp]),
    "moe_layer_forward": (_int, [_vp, _vp, _vp, _int, _vp, _vp, _vp, _vp, C.c_float, _vp]),
    "moe_gate_logits": (_int, [_vp, _int, _vp, _int, _int, _int, _vp, _vp, _vp, _vp]),
    "moe_rmsnorm": (_int, [_vp, _int, _int, _int, C.c_float, _vp, _vp]),
    "moe_grouped_gemm": (_int, [_vp] + [_int] * 8 + [_vp] * 6),
    "moe_grouped_gemm_wgrad": (_int, [_vp, _vp] + [_int] * 7 + [_vp] * 3 + [_int] * 4 + [_vp] * 2),
    "moe_grouped_ffn_backward_workspace_bytes": (_sz, [_int, _int, _int]),
    "moe_grouped_ffn_backward": (_int, [_vp, _vp] + [_int] * 7 + [_vp] * 6 + [_int] * 4 + [_vp] * 3 + [_sz, _vp]),
    "moe_unpermute_backward": (_int, [_vp] * 4 + [_int] * 4 + [_vp] * 3),
    "moe_w4_expert_bytes": (_sz, [_int, _int]),
    "moe_quantize_w4": (_int, [_vp] + [_int] * 4 + [_vp] * 2),
    "moe_dequantize_w4": (_int, [_vp] + [_int] * 4 + [_vp] * 2),
    "moe_grouped_gemm_w4": (_int, [_vp] + [_int] * 6 + [_vp] * 6),
    "moe_grouped_ffn_w4_workspace_bytes": (_sz, [_int, _int]),
    "moe_grouped_ffn_w4": (_int, [_vp] + [_int] * 6 + [_vp] * 7 + [_sz, _vp]),
    "ew_probe_stream": (_int, [_vp, _vp, _sz, _int, _vp]),
    "ew_probe_mfma_bf16": (_int, [_int, _int, _int, _vp, _vp]),
    "ew_tune_ffn": (None, [_int, _int, _int, _int, _int, _int, _int]),
    "ew_tune_route": (None, [_int]),
}


class PoolStats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("page_bytes", "bytes_virtual", "pages_mapped", "pages_free", "pages_parked", "pages_created",
                                          "pages_released", "pages_shared", "bytes_experts", "experts_loaded")] + \
               [("f_mem", C.c_double)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class LayerDesc(C.Structure):
    """ew_layer: what moe_layer_forward has to know about a layer."""
    _fields_ = [(n, _int) for n in ("dtype", "H", "I", "M", "k", "N", "P", "S", "renormalize", "T_max")] + \
               [(n, _vp) for n in ("Wg", "bias", "expert_map", "w13", "w2", "w13_shared", "w2_shared", "logits", "ids", "w", "slot",
                                   "counts", "offsets", "pair_of_row", "row_of_pair", "y", "ws_perm")] + \
               [("ws_perm_bytes", _sz), ("ws_ffn", _vp), ("ws_ffn_bytes", _sz)]


class EWError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{ERR_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def lib() -> C.CDLL:
    """The loaded library.  Raises if it has not been built (python -m paper_2508_17624_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2508_17624_amd.build`; "
                               "there is no fallback path")
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        _lib = l
    return _lib


def _check(rc: int):
    if rc != 0:
        raise EWError(rc, lib().ew_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream():
    # the raw handle: current_stream() builds a Stream object around it, five times the cost
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _type_code(dtype: torch.dtype) -> int:
    if dtype == torch.float32:
        return EW_F32
    if dtype == torch.bfloat16:
        return EW_BF16
    raise TypeError(f"unsupported dtype {dtype}")


def _dtype_code(t: torch.Tensor) -> int:
    return _type_code(t.dtype)


def _workspace(nbytes: int, device) -> torch.Tensor | None:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device) if nbytes else None


# ----------------------------------------------------------------------------- expert pool
class ExpertPool:
    """Owns an ew_pool*.  Weights handed to map() may be CPU or CUDA tensors (or None)."""

    def __init__(self, num_layers, M, N, E_max, w13_bytes, w2_bytes, page_bytes=0, prealloc_pages=0,
                 flags=EW_POOL_VMM, device=0):
        self._h = C.c_void_p()
        _check(lib().expert_pool_create(C.byref(self._h), device, num_layers, M, N, E_max, w13_bytes, w2_bytes,
                                        page_bytes, prealloc_pages, flags))
        self.L, self.M, self.N, self.E_max, self.P = num_layers, M, N, E_max, M + N * E_max
        self.w13_bytes, self.w2_bytes = w13_bytes, w2_bytes
        self.flags, self.device = flags, device
        self._keep = []

    @property
    def fake(self):
        return bool(self.flags & EW_POOL_FAKE)

    def close(self):
        if self._h:
            _check(lib().expert_pool_destroy(self._h))
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def map(self, layer, adapter_id, expert_ids, w13=None, w2=None, stream=None):
        ids = None
        n = 0
        if expert_ids is not None:
            ids = (C.c_int32 * len(expert_ids))(*[int(e) for e in expert_ids])
            n = len(expert_ids)
        for w, each in ((w13, self.w13_bytes), (w2, self.w2_bytes)):
            if w is not None and not w.is_contiguous():
                raise ValueError("weights must be contiguous")
            if w is not None and w.numel() * w.element_size() < n * each:
                raise ValueError(f"weights have {w.numel() * w.element_size()} bytes, {n} experts of {each} are needed")
        st = stream if stream is not None else (None if self.fake else _stream())
        _check(lib().expert_pool_map(self._h, layer, adapter_id, n, C.cast(ids, C.c_void_p) if ids is not None else None,
                                     _ptr(w13), _ptr(w2), st))
        if not self.fake:
            torch.cuda.current_stream().synchronize()      # host sources may be freed by the caller afterwards

    def unmap(self, layer, adapter_id):
        _check(lib().expert_pool_unmap(self._h, layer, adapter_id, None if self.fake else _stream()))

    def view(self, layer):
        """(w13_base, w2_base, expert_map_ptr, P) as integers."""
        a, b, m, p = C.c_void_p(), C.c_void_p(), C.c_void_p(), C.c_int()
        _check(lib().expert_pool_view(self._h, layer, C.byref(a), C.byref(b), C.byref(m), C.byref(p)))
        return a.value, b.value, m.value, p.value

    def expert_map_host(self, layer):
        out = torch.empty((self.N + 1, self.M), dtype=torch.int32)
        _check(lib().expert_pool_expert_map_host(self._h, layer, out.data_ptr()))
        return out

    def touch(self, adapter_ids):
        """Marks the adapters of a scheduled batch as just used (eviction order)."""
        ids = (C.c_int32 * len(adapter_ids))(*[int(a) for a in adapter_ids])
        _check(lib().expert_pool_touch(self._h, len(adapter_ids), ids))

    def lru_victim(self) -> int:
        """The loaded adapter used least recently, or -1."""
        out = C.c_int(-1)
        _check(lib().expert_pool_lru_victim(self._h, C.byref(out)))
        return out.value

    def stats(self) -> dict:
        s = PoolStats()
        _check(lib().expert_pool_stats(self._h, C.byref(s)))
        return s.as_dict()

    def trim(self, keep_pages=0):
        _check(lib().expert_pool_trim(self._h, keep_pages))

    def fake_fail_at(self, op, n):
        _check(lib().expert_pool_fake_fail_at(self._h, op, n))

    def fake_is_mapped(self, layer, which, offset) -> bool:
        out = C.c_int()
        _check(lib().expert_pool_fake_is_mapped(self._h, layer, which, offset, C.byref(out)))
        return bool(out.value)


# ----------------------------------------------------------------------------- hot path
def moe_route_topk(logits: torch.Tensor, k: int, renormalize: bool = False):
    T, E = logits.shape
    ids = torch.empty((T, k), dtype=torch.int32, device=logits.device)
    w = torch.empty((T, k), dtype=torch.float32, device=logits.device)
    _check(lib().moe_route_topk(_ptr(logits), T, E, k, int(renormalize), _ptr(ids), _ptr(w), _stream()))
    return ids, w


def moe_reroute_permute(topk_ids, adapter_id, expert_map, N: int, P: int, E: int | None = None, want_row_of_pair=True,
                        ws=None):
    """expert_map: int32 tensor [N+1, E] on the device, or a raw device pointer (then pass E)."""
    T, k = topk_ids.shape
    if E is None:
        E = expert_map.shape[1]
    dev = topk_ids.device
    slot = torch.empty((T, k), dtype=torch.int32, device=dev)
    counts = torch.empty(P, dtype=torch.int32, device=dev)
    offsets = torch.empty(P + 1, dtype=torch.int32, device=dev)
    por = torch.empty(T * k, dtype=torch.int32, device=dev)
    rop = torch.empty(T * k, dtype=torch.int32, device=dev) if want_row_of_pair else None
    need = lib().moe_reroute_permute_workspace_bytes(T, k, P)
    ws = ws if ws is not None else _workspace(need, dev)
    _check(lib().moe_reroute_permute(_ptr(topk_ids), _ptr(adapter_id), _ptr(expert_map), T, k, E, N, P, _ptr(slot),
                                     _ptr(counts), _ptr(offsets), _ptr(por), _ptr(rop), _ptr(ws),
                                     ws.numel() if ws is not None else 0, _stream()))
    return slot, counts, offsets, por, rop


def moe_reroute_permute_static(topk_ids, adapter_id, expert_map, N: int, P: int, out, E: int | None = None):
    """The variant that allocates nothing: `out` = (slot [T,k], counts [P], offsets [P+1], pair_of_row [T*k],
    row_of_pair [T*k] or None), all preallocated by the caller; scratch is the library's built-in buffer."""
    T, k = topk_ids.shape
    if E is None:
        E = expert_map.shape[1]
    slot, counts, offsets, por, rop = out
    _check(lib().moe_reroute_permute_static(_ptr(topk_ids), _ptr(adapter_id), _ptr(expert_map), T, k, E, N, P, _ptr(slot),
                                            _ptr(counts), _ptr(offsets), _ptr(por), _ptr(rop), _stream()))
    return out


def moe_route_reroute_permute(logits, adapter_id, expert_map, k: int, N: int, P: int, renormalize=False, ws=None):
    T, E = logits.shape
    dev = logits.device
    ids = torch.empty((T, k), dtype=torch.int32, device=dev)
    w = torch.empty((T, k), dtype=torch.float32, device=dev)
    slot = torch.empty((T, k), dtype=torch.int32, device=dev)
    counts = torch.empty(P, dtype=torch.int32, device=dev)
    offsets = torch.empty(P + 1, dtype=torch.int32, device=dev)
    por = torch.empty(T * k, dtype=torch.int32, device=dev)
    rop = torch.empty(T * k, dtype=torch.int32, device=dev)
    need = lib().moe_reroute_permute_workspace_bytes(T, k, P)
    ws = ws if ws is not None else _workspace(need, dev)
    _check(lib().moe_route_reroute_permute(_ptr(logits), _ptr(adapter_id), _ptr(expert_map), T, E, k, N, P,
                                           int(renormalize), _ptr(ids), _ptr(w), _ptr(slot), _ptr(counts), _ptr(offsets),
                                           _ptr(por), _ptr(rop), _ptr(ws), ws.numel() if ws is not None else 0,
                                           _stream()))
    return ids, w, slot, counts, offsets, por, rop


def moe_reroute_singleop(topk_ids, adapter_id, expert_map, N: int, ws=None, out=None):
    """The unfused rerouting baseline (three launches); returns slot_ids [T, k]."""
    T, k = topk_ids.shape
    E = expert_map.shape[1]
    slot = out if out is not None else torch.empty((T, k), dtype=torch.int32, device=topk_ids.device)
    ws = ws if ws is not None else _workspace(lib().moe_reroute_singleop_workspace_bytes(T, k), topk_ids.device)
    _check(lib().moe_reroute_singleop(_ptr(topk_ids), _ptr(adapter_id), _ptr(expert_map), T, k, E, N, _ptr(slot), _ptr(ws),
                                      ws.numel() if ws is not None else 0, _stream()))
    return slot


def moe_grouped_ffn(x, k: int, I: int, P: int, counts, offsets, pair_of_row, w13_base, w2_base, ws=None, out=None,
                    num_rows: int | None = None):
    """w13_base / w2_base: device tensors [P, 2I, H] / [P, H, I] or raw device pointers (pool views).
    num_rows = offsets[P], the number of sorted rows; defaults to x.shape[0] * k.  It differs from
    that only when rows do not come from a top-k (shared experts: num_rows = S * T with k = 1)."""
    H = x.shape[1]
    rows = x.shape[0] * k if num_rows is None else num_rows
    if rows % k:
        raise ValueError("num_rows must be a multiple of k")
    T = rows // k
    dt = _dtype_code(x)
    y = out if out is not None else torch.empty((rows, H), dtype=x.dtype, device=x.device)
    if y.shape[0] < rows:
        raise ValueError("output has fewer rows than num_rows")
    need = lib().moe_grouped_ffn_workspace_bytes(T, k, H, I, P, dt)
    ws = ws if ws is not None else _workspace(need, x.device)
    _check(lib().moe_grouped_ffn(_ptr(x), dt, T, k, H, I, P, _ptr(counts), _ptr(offsets), _ptr(pair_of_row),
                                 _ptr(w13_base), _ptr(w2_base), _ptr(y), _ptr(ws), ws.numel() if ws is not None else 0,
                                 _stream()))
    return y


def moe_grouped_ffn_with_shared(x, k: int, I: int, P: int, counts, offsets, pair_of_row, w13_base, w2_base, w13_shared,
                                w2_shared, ws=None, out=None):
    """Routed and shared experts in one call.  w13_shared / w2_shared: [S, 2I, H] / [S, H, I].  Returns y [T*(k+S), H]:
    the routed rows, then the shared experts' [S, T, H] outputs (y[T*k:] is moe_unpermute's shared_out)."""
    T, H = x.shape
    S = w13_shared.shape[0]
    dt = _dtype_code(x)
    rows = T * (k + S)
    y = out if out is not None else torch.empty((rows, H), dtype=x.dtype, device=x.device)
    if y.shape[0] < rows:
        raise ValueError("output has fewer than T*(k+S) rows")
    need = lib().moe_grouped_ffn_workspace_bytes(T, k + S, H, I, P + S, dt)
    ws = ws if ws is not None else _workspace(need, x.device)
    _check(lib().moe_grouped_ffn_with_shared(_ptr(x), dt, T, k, H, I, P, S, _ptr(counts), _ptr(offsets), _ptr(pair_of_row),
                                             _ptr(w13_base), _ptr(w2_base), _ptr(w13_shared), _ptr(w2_shared), _ptr(y),
                                             _ptr(ws), ws.numel() if ws is not None else 0, _stream()))
    return y


def moe_unpermute(y_sorted, row_of_pair, topk_w, shared_out=None, out=None, residual=None):
    """shared_out: [S, T, H] (or [S*T, H]) slabs of shared-expert outputs, or None; residual: [T, H] or None."""
    T, k = topk_w.shape
    H = y_sorted.shape[1]
    S = 0 if shared_out is None else shared_out.numel() // (T * H)
    o = out if out is not None else torch.empty((T, H), dtype=y_sorted.dtype, device=y_sorted.device)
    _check(lib().moe_unpermute(_ptr(y_sorted), _ptr(row_of_pair), _ptr(topk_w), _ptr(shared_out), S, _ptr(residual), T, k, H,
                               _dtype_code(y_sorted), _ptr(o), _stream()))
    return o


def moe_unpermute_rmsnorm(y_sorted, row_of_pair, topk_w, eps: float, shared_out=None, out=None, normed_out=None, residual=None):
    """moe_unpermute and moe_rmsnorm of its result in one launch; returns (out, normed_out)."""
    T, k = topk_w.shape
    H = y_sorted.shape[1]
    S = 0 if shared_out is None else shared_out.numel() // (T * H)
    o = out if out is not None else torch.empty((T, H), dtype=y_sorted.dtype, device=y_sorted.device)
    n = normed_out if normed_out is not None else torch.empty_like(o)
    _check(lib().moe_unpermute_rmsnorm(_ptr(y_sorted), _ptr(row_of_pair), _ptr(topk_w), _ptr(shared_out), S, _ptr(residual), T, k,
                                       H, _dtype_code(y_sorted), _ptr(o), eps, _ptr(n), _stream()))
    return o, n


def tune_ffn(path: int = 0, stream_token_tiles: int = 0, stream_threads: int = 0, ws_frags: int = 0,
             ws_chunk_frags: int = 0, ws_wait_ticks: int = -1, ws_two_launches: bool = False):
    """Kernel-selection override of moe_grouped_ffn(bf16), process-global; no arguments = automatic.
    path 1 = register-streaming kernel (stream_token_tiles 1|2, stream_threads), 2 = LDS-tiled GEMM kernel,
    3 = LDS-direct kernels (ws_frags 1|2|4|8 = kernel shape, ws_chunk_frags = cap on 32-row fragments
    per row chunk, ws_two_launches = the two products as two launches, ws_wait_ticks > 0 = looks before a unit of the second
    product gives up waiting for its activation rows and writes NaN)."""
    lib().ew_tune_ffn(path, stream_token_tiles, stream_threads, ws_frags, ws_chunk_frags, ws_wait_ticks, int(ws_two_launches))


def tune_route(small_pairs: int = 2048):
    """Pairs (T*k) up to which moe_reroute_permute / moe_route_reroute_permute take the single-block permutation
    (with the router fused and few tokens that block selects too, otherwise a multi-block top-k kernel runs before it)."""
    lib().ew_tune_route(small_pairs)


def moe_gate_logits(x, Wg, adapter_id=None, bias=None):
    T, H = x.shape
    E = Wg.shape[0]
    logits = torch.empty((T, E), dtype=torch.float32, device=x.device)
    _check(lib().moe_gate_logits(_ptr(x), _dtype_code(x), _ptr(Wg), T, H, E, _ptr(adapter_id), _ptr(bias), _ptr(logits),
                                 _stream()))
    return logits


def moe_rmsnorm(x, eps: float = 1e-6, out=None):
    T, H = x.shape
    o = out if out is not None else torch.empty_like(x)
    _check(lib().moe_rmsnorm(_ptr(x), _dtype_code(x), T, H, float(eps), _ptr(o), _stream()))
    return o


# ----------------------------------------------------------------------------- the experts' products one by one
def _need(name, t, dtype, numel, like):
    """Checks an operand: a contiguous tensor of this type on the device of `like`, with room for numel elements; or a raw
    device pointer (a pool's tensor), or None."""
    if t is None or isinstance(t, int):
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, is {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.get_device() != like.get_device():  # (numbers: comparing devices takes twice as long)
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")
    if t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, {numel} are needed")


def _current(x):
    """The device of x, which has to be the current one: kernels are enqueued on its current stream."""
    if not x.is_cuda or x.get_device() != torch.cuda.current_device():
        raise ValueError(f"tensors are on {x.device}, not on the current HIP device")
    return x.device


def _fits(*sizes):
    """The library counts in 32 bits; a larger number would reach it as another one."""
    if max(sizes) >= 2 ** 31:
        raise ValueError(f"sizes and row counts must be below 2^31, got {max(sizes)}")


def _sorted_rows(x, k, P, counts, offsets, pair_of_row, num_rows, width):
    """Number of sorted rows of a call, after checking what names them; width: its other size."""
    if x.dim() != 2 or not x.is_contiguous():
        raise ValueError("token rows must be a contiguous 2-D tensor")
    rows = x.shape[0] * k if num_rows is None else num_rows
    _fits(*x.shape, rows, k, P, width)
    _current(x)
    if pair_of_row is None and rows > x.shape[0] * k:
        raise ValueError("more rows than pairs")
    _need("counts", counts, torch.int32, P, x)
    _need("offsets", offsets, torch.int32, P + 1, x)
    _need("pair_of_row", pair_of_row, torch.int32, rows, x)
    return rows


def _result(name, out, shape, dtype, like):
    if out is None:
        return like.new_empty(shape, dtype=dtype)  # (two thirds of torch.empty's time)
    n = 1
    for d in shape:
        n *= d
    _need(name, out, dtype, n, like)
    return out


def _scratch(ws, need, like):
    if ws is None:
        return _workspace(need, like.device)
    _need("workspace", ws, torch.uint8, 0, like)
    return ws


def moe_grouped_gemm(x, k: int, N: int, P: int, counts, offsets, pair_of_row, w_base, transposed=False, out=None,
                     num_rows: int | None = None):
    """y[r] = W_s x[pair_of_row[r] / k] for the rows r of every slot s, w_base [P, N, K]; transposed: W_s^T, w_base [P, K, N] (the
    input gradient: x = dy, k = 1, pair_of_row None).  w_base: a tensor or a raw device pointer (pool view).
    num_rows defaults to x.shape[0] * k; returns y [num_rows, N], rows behind the last one as they were."""
    rows, K = _sorted_rows(x, k, P, counts, offsets, pair_of_row, num_rows, N), x.shape[1]
    _need("w_base", w_base, x.dtype, P * N * K, x)
    y = _result("out", out, (rows, N), x.dtype, x)
    _check(lib().moe_grouped_gemm(_ptr(x), _dtype_code(x), x.shape[0], rows, k, K, N, P, int(transposed), _ptr(counts), _ptr(offsets),
                                  _ptr(pair_of_row), _ptr(w_base), _ptr(y), _stream()))
    return y


def moe_grouped_gemm_wgrad(dy, x, k: int, P: int, counts, offsets, pair_of_row, first_slot: int = 0, num_slots: int | None = None,
                           dtype=torch.float32, accumulate=False, out=None):
    """dW [num_slots, N, K] of moe_grouped_gemm from dy [rows, N] (sorted rows) and x [*, K], for the slots from first_slot on (all by
    default); accumulate adds to `out` (float32)."""
    if dy.dim() != 2 or not dy.is_contiguous() or dy.dtype != x.dtype or dy.device != x.device:
        raise ValueError("dy must be a contiguous 2-D tensor of x's type and device")
    dw_code = _type_code(dtype)
    n = P - first_slot if num_slots is None else num_slots
    _fits(abs(first_slot), abs(n))
    rows, K, N = _sorted_rows(x, k, P, counts, offsets, pair_of_row, dy.shape[0], dy.shape[1]), x.shape[1], dy.shape[1]
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    dw = _result("out", out, (max(n, 0), N, K), dtype, x)
    _check(lib().moe_grouped_gemm_wgrad(_ptr(dy), _ptr(x), _dtype_code(x), x.shape[0], rows, k, K, N, P, _ptr(counts), _ptr(offsets), _ptr(pair_of_row),
                                        first_slot, n, dw_code, int(accumulate), _ptr(dw), _stream()))
    return dw


def moe_grouped_ffn_backward(x, dy, k: int, I: int, P: int, counts, offsets, pair_of_row, w13_base, w2_base, first_slot: int = 0,
                             num_slots: int | None = None, dw_dtype=torch.float32, accumulate=False, want_dx=True, ws=None, dx=None,
                             dw13=None, dw2=None):
    """Gradients of moe_grouped_ffn from dy [rows, H]: (dx_sorted [rows, H], dw13 [num_slots, 2I, H], dw2 [num_slots, H, I]) for the
    slots from first_slot on (all by default; num_slots = 0: none, then the weight gradients are None).  accumulate adds to dw13
    and dw2 (float32).  A token's input gradient: moe_unpermute(dx_sorted, row_of_pair, ones)."""
    if dy.dim() != 2 or not dy.is_contiguous() or dy.dtype != x.dtype or dy.device != x.device or dy.shape[1] != x.shape[1]:
        raise ValueError("dy must be a contiguous [rows, H] tensor of x's type and device")
    dw_code = _type_code(dw_dtype)
    n = P - first_slot if num_slots is None else num_slots
    _fits(abs(first_slot), abs(n))
    rows, H = _sorted_rows(x, k, P, counts, offsets, pair_of_row, dy.shape[0], 2 * I), x.shape[1]
    if accumulate and (dw13 is None or dw2 is None):
        raise ValueError("accumulate needs dw13 and dw2")
    _need("w13_base", w13_base, x.dtype, P * 2 * I * H, x)
    _need("w2_base", w2_base, x.dtype, P * H * I, x)
    dx = _result("dx", dx, (rows, H), x.dtype, x) if want_dx else None
    if n > 0:
        dw13 = _result("dw13", dw13, (n, 2 * I, H), dw_dtype, x)
        dw2 = _result("dw2", dw2, (n, H, I), dw_dtype, x)
    else:
        dw13 = dw2 = None
    ws = _scratch(ws, lib().moe_grouped_ffn_backward_workspace_bytes(rows, I, _dtype_code(x)), x)
    _check(lib().moe_grouped_ffn_backward(_ptr(x), _ptr(dy), _dtype_code(x), x.shape[0], rows, k, H, I, P, _ptr(counts), _ptr(offsets), _ptr(pair_of_row),
                                          _ptr(w13_base), _ptr(w2_base), _ptr(dx), first_slot, n, dw_code, int(accumulate),
                                          _ptr(dw13), _ptr(dw2), _ptr(ws), ws.numel() if ws is not None else 0, _stream()))
    return dx, dw13, dw2


def moe_unpermute_backward(dout, row_of_pair, topk_w, y_sorted=None, out=None, dw_out=None):
    """Gradients of moe_unpermute from dout [T, H]: (dy_sorted [T*k, H], dw [T, k]); dw is None without y_sorted."""
    T, k = topk_w.shape
    if dout.dim() != 2 or not dout.is_contiguous() or dout.shape[0] != T:
        raise ValueError("dout must be a contiguous [T, H] tensor")
    H = dout.shape[1]
    _fits(T * k, H)
    _current(dout)
    _need("row_of_pair", row_of_pair, torch.int32, T * k, dout)
    _need("topk_w", topk_w, torch.float32, T * k, dout)
    _need("y_sorted", y_sorted, dout.dtype, T * k * H, dout)
    dy = _result("out", out, (T * k, H), dout.dtype, dout)
    dw = _result("dw_out", dw_out, (T, k), torch.float32, dout) if y_sorted is not None else None
    _check(lib().moe_unpermute_backward(_ptr(dout), _ptr(y_sorted), _ptr(row_of_pair), _ptr(topk_w), T, k, H, _dtype_code(dout), _ptr(dy),
                                        _ptr(dw), _stream()))
    return dy, dw


# ----------------------------------------------------------------------------- experts in 4 bits
def moe_w4_expert_bytes(N: int, K: int) -> int:
    """Bytes of an expert's [N, K] weights in 4 bits: codes [N, K/2], then scales [N, K/32].  Also the size that ExpertPool takes for
    a pool of such experts.  Raises for sizes that cannot be packed."""
    _fits(N, K)
    n = lib().moe_w4_expert_bytes(N, K)
    if n == 0:
        raise EWError(-6, f"K must be a multiple of 32 and N*K of 512 (N={N} K={K})")
    return n


def moe_quantize_w4(w, out=None):
    """w [E, N, K] (float32 or bfloat16) -> uint8 [E, moe_w4_expert_bytes(N, K)], what ExpertPool.map takes for a 4-bit pool."""
    if w.dim() != 3 or not w.is_contiguous():
        raise ValueError("w must be a contiguous [experts, N, K] tensor")
    E, N, K = w.shape
    _fits(E, N, K)
    _current(w)
    o = _result("out", out, (E, moe_w4_expert_bytes(N, K)), torch.uint8, w)
    _check(lib().moe_quantize_w4(_ptr(w), _dtype_code(w), E, N, K, _ptr(o), _stream()))
    return o


def moe_dequantize_w4(w4, N: int, K: int, dtype=torch.bfloat16, out=None):
    """The values that packed experts uint8 [E, moe_w4_expert_bytes(N, K)] stand for, [E, N, K]."""
    if w4.dim() != 2 or not w4.is_contiguous() or w4.dtype != torch.uint8 or w4.shape[1] != moe_w4_expert_bytes(N, K):
        raise ValueError("w4 must be a contiguous uint8 [experts, moe_w4_expert_bytes(N, K)] tensor")
    _current(w4)
    o = _result("out", out, (w4.shape[0], N, K), dtype, w4)
    _check(lib().moe_dequantize_w4(_ptr(w4), _dtype_code(o), w4.shape[0], N, K, _ptr(o), _stream()))
    return o


def moe_grouped_gemm_w4(x, k: int, N: int, P: int, counts, offsets, pair_of_row, w4_base, out=None, num_rows: int | None = None):
    """moe_grouped_gemm with 4-bit experts: w4_base uint8 [P, moe_w4_expert_bytes(N, K)] or a raw device pointer; x bfloat16."""
    if x.dtype != torch.bfloat16:
        raise TypeError(f"token rows of 4-bit experts are bfloat16, not {x.dtype}")
    rows, K = _sorted_rows(x, k, P, counts, offsets, pair_of_row, num_rows, N), x.shape[1]
    _need("w4_base", w4_base, torch.uint8, P * moe_w4_expert_bytes(N, K), x)
    y = _result("out", out, (rows, N), x.dtype, x)
    _check(lib().moe_grouped_gemm_w4(_ptr(x), x.shape[0], rows, k, K, N, P, _ptr(counts), _ptr(offsets), _ptr(pair_of_row), _ptr(w4_base), _ptr(y), _stream()))
    return y


def moe_grouped_ffn_w4(x, k: int, I: int, P: int, counts, offsets, pair_of_row, w13_base, w2_base, ws=None, out=None,
                       num_rows: int | None = None):
    """moe_grouped_ffn with 4-bit experts: w13_base uint8 [P, moe_w4_expert_bytes(2I, H)], w2_base uint8 [P, moe_w4_expert_bytes(H, I)],
    or raw device pointers (pool views); x bfloat16."""
    if x.dtype != torch.bfloat16:
        raise TypeError(f"token rows of 4-bit experts are bfloat16, not {x.dtype}")
    rows, H = _sorted_rows(x, k, P, counts, offsets, pair_of_row, num_rows, 2 * I), x.shape[1]
    _need("w13_base", w13_base, torch.uint8, P * moe_w4_expert_bytes(2 * I, H), x)
    _need("w2_base", w2_base, torch.uint8, P * moe_w4_expert_bytes(H, I), x)
    y = _result("out", out, (rows, H), x.dtype, x)
    ws = _scratch(ws, lib().moe_grouped_ffn_w4_workspace_bytes(rows, I), x)
    _check(lib().moe_grouped_ffn_w4(_ptr(x), x.shape[0], rows, k, H, I, P, _ptr(counts), _ptr(offsets), _ptr(pair_of_row), _ptr(w13_base), _ptr(w2_base),
                                    _ptr(y), _ptr(ws), ws.numel() if ws is not None else 0, _stream()))
    return y
