"""Thin ctypes binding of libbsa.so: argument marshalling only.

Every step of the request path (mask state, plan selection, launch preparation,
attention, Split-K merge) runs inside the C-ABI library; torch is used here only
to own device memory and streams.  Loading fails loudly if the library has not
been built -- there is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from typing import Dict, List, Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbsa.so")

BSA_OK = 0
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "NO_ELIGIBLE_PLAN", 4: "OOM", 5: "CUDA",
                6: "DEVICE_TIMEOUT", 7: "LUT"}
MAP_NAMES = {0: "direct", 1: "coarsened", 2: "refined"}


class PlanDesc(ctypes.Structure):
    _fields_ = [("plan_id", ctypes.c_int32), ("T_Q", ctypes.c_int32), ("T_KV", ctypes.c_int32),
                ("stages", ctypes.c_int32), ("split_tau", ctypes.c_int32), ("split_pmax", ctypes.c_int32),
                ("order", ctypes.c_int32), ("kernel", ctypes.c_int32), ("name", ctypes.c_char * 48)]


DTYPES = {"bf16": 0, "fp16": 1}  # BSA_DTYPE_*
LAYOUTS = {"hnd": 0, "nhd": 1}   # BSA_LAYOUT_*: [heads, N, d] or [N, heads, d]


class Options(ctypes.Structure):
    _fields_ = [("force_plan_id", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("max_workspace_bytes", ctypes.c_int64), ("N_kv", ctypes.c_int64),
                ("layout", ctypes.c_int32), ("batch", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("plan", PlanDesc), ("map_q", ctypes.c_int32), ("map_kv", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("d", ctypes.c_int32), ("B_Q", ctypes.c_int32), ("B_KV", ctypes.c_int32),
                ("N", ctypes.c_int64),
                ("nQb", ctypes.c_int32), ("nKb", ctypes.c_int32), ("nQt", ctypes.c_int32), ("nKt", ctypes.c_int32),
                ("member_bits", ctypes.c_int32), ("lut_hit", ctypes.c_int32), ("regime_bucket", ctypes.c_int32 * 4),
                ("nnz_blocks", ctypes.c_int64), ("blocks_in_runs", ctypes.c_int64),
                ("max_row_nnz", ctypes.c_int32), ("member_words", ctypes.c_int32),
                ("density", ctypes.c_double), ("run_coverage", ctypes.c_double), ("skew", ctypes.c_double),
                ("ntiles", ctypes.c_int64), ("nitems", ctypes.c_int64), ("nsplit_rows", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_int64), ("covered_pairs", ctypes.c_int64),
                ("us_mask_state", ctypes.c_float), ("us_stats_sync", ctypes.c_float), ("us_lookup", ctypes.c_float),
                ("us_launch_prep", ctypes.c_float), ("us_total", ctypes.c_float), ("device_status", ctypes.c_int32),
                ("N_kv", ctypes.c_int64), ("dtype", ctypes.c_int32), ("layout", ctypes.c_int32)]

    def as_dict(self) -> Dict:
        out = {}
        for name, _ in self._fields_:
            v = getattr(self, name)
            if name == "plan":
                v = {f: (getattr(v, f).decode() if f == "name" else getattr(v, f)) for f, _ in PlanDesc._fields_}
            elif name == "regime_bucket":
                v = list(v)
            out[name] = v
        return out


_lib = None


def lib() -> ctypes.CDLL:
    """Load libbsa.so (raises if it was not built: there is no other code path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_25869_b200.build` "
                           "(nvcc, sm_100a). There is no CPU or PyTorch fallback.")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_double
    L.bsa_plan_create.argtypes = [vp, i32, i32, i64, i32, i32, ctypes.POINTER(vp)]
    L.bsa_plan_create_ex.argtypes = [vp, i32, i32, i64, i32, i32, ctypes.POINTER(Options), vp, ctypes.POINTER(vp)]
    L.bsa_plan_create_packed.argtypes = [vp, i64, i32, i32, i64, i32, i32, ctypes.POINTER(Options), vp, ctypes.POINTER(vp)]
    L.bsa_plan_cache_create.argtypes = [i32, ctypes.POINTER(vp)]
    L.bsa_plan_cache_get.argtypes = [vp, vp, i64, i32, i32, i64, i32, i32, ctypes.POINTER(Options), vp, ctypes.POINTER(vp),
                                     ctypes.POINTER(i32)]
    L.bsa_plan_cache_request.argtypes = [vp, vp, i64, i32, i32, i64, i32, i32, vp, vp, vp, vp, vp, ctypes.POINTER(Options),
                                         vp, ctypes.POINTER(vp), ctypes.POINTER(i32)]
    L.bsa_plan_cache_stats.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64),
                                       ctypes.POINTER(ctypes.c_int32)]
    L.bsa_plan_cache_destroy.argtypes = [vp]
    L.bsa_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.bsa_request_device.argtypes = [vp, i64, i32, i32, i64, i32, i32, vp, vp, vp, vp, vp, ctypes.POINTER(Options), vp,
                                     ctypes.POINTER(vp)]
    L.bsa_plan_destroy.argtypes = [vp]
    L.bsa_request_host.argtypes = [vp, i32, i32, i64, i32, i32, vp, vp, vp, vp, vp, ctypes.POINTER(Options),
                                   ctypes.POINTER(PlanInfo)]
    L.bsa_mask_stats_noalloc.argtypes = [vp, i32, i32, i32, vp, vp]
    L.bsa_rope.argtypes = [ctypes.c_char_p] * 5 + [vp]
    L.bsa_window_forward.argtypes = [ctypes.c_char_p] * 5 + [vp, vp]
    L.bsa_window_backward.argtypes = [ctypes.c_char_p] * 5 + [vp] + [ctypes.c_char_p] * 4 + [vp, i64, vp]
    L.bsa_window_workspace_bytes.argtypes = [ctypes.c_char_p]
    L.bsa_window_workspace_bytes.restype = i64
    L.bsa_window_status.argtypes = [ctypes.POINTER(ctypes.c_int)]
    L.bsa_plan_get_info.argtypes = [vp, ctypes.POINTER(PlanInfo)]
    L.bsa_plan_export_csr.argtypes = [vp, vp, vp]
    L.bsa_plan_export_tiles.argtypes = [vp, i32, vp, vp, vp, i64, ctypes.POINTER(i64)]
    L.bsa_plan_export_items.argtypes = [vp, vp, i64, ctypes.POINTER(i64)]
    L.bsa_catalog_size.restype = i32
    L.bsa_catalog_get.argtypes = [i32, ctypes.POINTER(PlanDesc)]
    L.bsa_plan_eligible.argtypes = [i32, i32, i32, i64, i32, i32, i64]
    L.bsa_plan_eligible_ex.argtypes = [i32, i32, i32, i64, i64, i32, i32, i32, i64]
    L.bsa_debug_set_wait_limit.argtypes = [ctypes.c_longlong]
    L.bsa_debug_withhold_arrival.argtypes = [i32]
    L.bsa_debug_merge_only.argtypes = [vp, vp, vp, vp]
    L.bsa_base_plan.argtypes = [i32, i32, i32]
    L.bsa_catalog_hash.restype = ctypes.c_uint64
    L.bsa_lut_load.argtypes = [ctypes.c_char_p]
    L.bsa_lut_clear.restype = None
    L.bsa_lut_select.argtypes = [i32, i32, i64, i32, i32, f64, f64, f64, i64, ctypes.POINTER(i32)]
    L.bsa_lut_buckets.argtypes = [i64, f64, f64, f64, ctypes.POINTER(ctypes.c_int32)]
    L.bsa_lut_buckets.restype = None
    L.bsa_force_plan.argtypes = [i32]
    L.bsa_force_plan.restype = None
    L.bsa_status_string.argtypes = [i32]
    L.bsa_status_string.restype = ctypes.c_char_p
    L.bsa_last_cuda_error.restype = ctypes.c_char_p
    L.bsa_version.restype = ctypes.c_char_p
    L.bsa_kernel_launch_count.restype = i64
    _lib = L
    load_default_table()
    return L


DEFAULT_TABLE = os.path.join(_HERE, "plan_table_b200.lut")


def load_default_table() -> bool:
    """Load the plan table shipped with the package (written by ``lut_build.py`` on a B200).  A table built
    for another catalog is rejected by the library; base plans are used then.  Returns True if loaded."""
    if _lib is None or not os.path.exists(DEFAULT_TABLE):
        return False
    return _lib.bsa_lut_load(DEFAULT_TABLE.encode()) == BSA_OK


class BsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = lib().bsa_last_cuda_error().decode() if status == 5 else ""
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} "
                         f"({lib().bsa_status_string(status).decode()}) {detail}")


def _check(status: int, where: str):
    if status != BSA_OK:
        raise BsaError(status, where)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        # the handle alone: building a Stream object around it takes 3 us of a forward's 14
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    return getattr(stream, "cuda_stream", stream) or None


def _pool(stream, dev: int):
    """Context in which a call on ``stream`` (a torch stream or a handle) allocates: its memory comes from that stream's pool.  From the
    current stream's it could be memory that work queued there is still using, and be handed out again while ``stream`` writes it."""
    import torch
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream_ptr(stream)
        stream = torch.cuda.ExternalStream(handle, device=dev) if handle else torch.cuda.default_stream(dev)
    return torch.cuda.stream(stream)


def _lse_shape(Q, layout: str):
    """[heads, N] for Q stored [heads, N, d], [N, heads, d] or, batched and token-major, [batch, N, heads/batch, d]."""
    if layout == "hnd":
        return (Q.shape[0], Q.shape[1]) if Q.dim() == 3 else (Q.shape[0] * Q.shape[1], Q.shape[2])
    if Q.dim() == 4:
        return (Q.shape[0] * Q.shape[2], Q.shape[1])
    return (Q.shape[1], Q.shape[0])


def _fresh_outputs(Q, layout: str, O, LSE, stream):
    """O and LSE of a plan's forward, those that are None allocated where ``stream`` (None: the current one) writes them."""
    import torch
    if stream is not None:
        with _pool(stream, Q.get_device()):
            return _fresh_outputs(Q, layout, O, LSE, None)
    if O is None:
        O = torch.empty_like(Q)
    if LSE is None:  # [heads, N] whatever the layout of Q
        LSE = Q.new_empty(_lse_shape(Q, layout), dtype=torch.float32)
    return O, LSE


class Plan:
    """Handle of a prepared plan (``bsa_plan_create`` ... ``bsa_plan_destroy``)."""

    def __init__(self, handle: int, layout: str = "hnd"):
        self._h = ctypes.c_void_p(handle)
        self.layout = layout

    def forward(self, Q, K, V, O=None, LSE=None, stream=None):
        """``bsa_forward``: Q, K, V are bf16 CUDA tensors ``[heads, N, d]``; returns ``(O, LSE)``.  ``stream``: a torch stream or a
        handle; fresh outputs come from its pool, as if allocated with it current."""
        import torch
        assert Q.is_cuda and Q.dtype in (torch.bfloat16, torch.float16) and Q.is_contiguous()  # as the plan's dtype
        assert K.is_contiguous() and V.is_contiguous() and K.dtype == V.dtype == Q.dtype
        if O is None or LSE is None:
            O, LSE = _fresh_outputs(Q, self.layout, O, LSE, stream)
        _check(lib().bsa_forward(self._h, Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), LSE.data_ptr(),
                                 _stream_ptr(stream)), "bsa_forward")
        return O, LSE

    def merge_only(self, O, LSE, stream=None):
        """``bsa_debug_merge_only`` (measurement hook): the Split-K reduction kernel alone, over the last forward's partials."""
        _check(lib().bsa_debug_merge_only(self._h, O.data_ptr(), LSE.data_ptr(), _stream_ptr(stream)), "bsa_debug_merge_only")

    def info(self) -> Dict:
        inf = PlanInfo()
        _check(lib().bsa_plan_get_info(self._h, ctypes.byref(inf)), "bsa_plan_get_info")
        return inf.as_dict()

    def export_csr(self) -> Tuple[np.ndarray, np.ndarray]:
        inf = self.info()
        rp = np.zeros(inf["heads"] * inf["nQb"] + 1, dtype=np.int32)
        ci = np.zeros(max(1, inf["nnz_blocks"]), dtype=np.int32)
        _check(lib().bsa_plan_export_csr(self._h, rp.ctypes.data, ci.ctypes.data), "bsa_plan_export_csr")
        return rp, ci[: inf["nnz_blocks"]]

    def export_tiles(self, head: int):
        """Tiles of one head: ``(tile_row_ptr [nQt+1], tile_col [n], tile_member [n, W] uint64)`` with
        ``W = T_Q / 128`` membership words per tile (one per 128-row slot)."""
        n = ctypes.c_int64(0)
        _check(lib().bsa_plan_export_tiles(self._h, head, None, None, None, 0, ctypes.byref(n)), "export_tiles(size)")
        inf = self.info()
        nQt, W = inf["nQt"], inf["member_words"]
        rp = np.zeros(nQt + 1, dtype=np.int32)
        tc = np.zeros(max(1, n.value), dtype=np.int32)
        tm = np.zeros((max(1, n.value), W), dtype=np.uint64)
        _check(lib().bsa_plan_export_tiles(self._h, head, rp.ctypes.data, tc.ctypes.data, tm.ctypes.data,
                                           max(1, n.value), ctypes.byref(n)), "export_tiles")
        return rp, tc[: n.value], tm[: n.value]

    def export_items(self) -> np.ndarray:
        n = ctypes.c_int64(0)
        _check(lib().bsa_plan_export_items(self._h, None, 0, ctypes.byref(n)), "export_items(size)")
        it = np.zeros((max(1, n.value), 8), dtype=np.int32)
        _check(lib().bsa_plan_export_items(self._h, it.ctypes.data, max(1, n.value), ctypes.byref(n)), "export_items")
        return it[: n.value]

    def destroy(self):
        if self._h:
            _check(lib().bsa_plan_destroy(self._h), "bsa_plan_destroy")
            self._h = None

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.destroy()


def plan_create(mask, B_Q: int, B_KV: int, N: int, heads: int, d: int, plan_id: int = -1,
                max_workspace_bytes: int = 0, stream=None, N_kv: int = 0, dtype: str = "bf16",
                layout: str = "hnd", batch: int = 0) -> Plan:
    """``bsa_plan_create_ex``: ``mask`` is a uint8/bool CUDA tensor ``[heads, nQb, nKb]``; ``N_kv`` > 0 gives K and V
    that many tokens per head (Q, O, LSE keep ``N``); ``dtype`` "fp16" prepares the plan for half tensors; ``batch`` > 1
    with ``layout="nhd"`` makes the tensors ``[batch, N, heads / batch, d]`` (``heads`` counts all problems)."""
    import torch
    assert mask.is_cuda and mask.is_contiguous() and mask.dtype in (torch.uint8, torch.bool)
    h = ctypes.c_void_p()
    opt = Options(plan_id, DTYPES[dtype], max_workspace_bytes, N_kv, LAYOUTS[layout], batch)
    _check(lib().bsa_plan_create_ex(mask.data_ptr(), B_Q, B_KV, N, heads, d, ctypes.byref(opt), _stream_ptr(stream),
                                    ctypes.byref(h)), "bsa_plan_create")
    return Plan(h.value, layout)


def request(mask, B_Q: int, B_KV: int, N: int, heads: int, d: int, Q, K, V, O=None, LSE=None, plan_id: int = -1,
            max_workspace_bytes: int = 0, stream=None, N_kv: int = 0, dtype: str = "bf16", layout: str = "hnd",
            row_stride: int = 0):
    """``bsa_request_device``: plan create + forward in one call (CUDA tensors).  Returns ``(plan, O, LSE)``; the plan
    can run further forwards and is given back with ``plan.destroy()``.  ``stream``: as for ``Plan.forward``."""
    if O is None or LSE is None:
        O, LSE = _fresh_outputs(Q, layout, O, LSE, stream)
    h = ctypes.c_void_p()
    opt = Options(plan_id, DTYPES[dtype], max_workspace_bytes, N_kv, LAYOUTS[layout], 0)
    _check(lib().bsa_request_device(mask.data_ptr(), row_stride, B_Q, B_KV, N, heads, d, Q.data_ptr(), K.data_ptr(),
                                    V.data_ptr(), O.data_ptr(), LSE.data_ptr(), ctypes.byref(opt), _stream_ptr(stream),
                                    ctypes.byref(h)), "bsa_request_device")
    return Plan(h.value, layout), O, LSE


def pack_mask(mask):
    """Bit-pack a uint8/bool mask tensor ``[heads, nQb, nKb]`` (CUDA or CPU) into the layout ``plan_create_packed``
    reads: little-endian bits, rows padded to a multiple of 4 bytes.  Returns ``(packed uint8 tensor, row stride)``.
    A convenience for callers and tests (plain torch ops, not part of the timed path)."""
    import torch
    h, nq, nk = mask.shape
    stride = ((nk + 31) // 32) * 4
    m = (mask != 0).to(torch.uint8)
    pad = stride * 8 - nk
    if pad:
        m = torch.nn.functional.pad(m, (0, pad))
    w = torch.tensor([1, 2, 4, 8, 16, 32, 64, 128], dtype=torch.uint8, device=m.device)
    packed = (m.view(h, nq, stride, 8) * w).sum(dim=-1, dtype=torch.int32).to(torch.uint8).contiguous()
    return packed, stride


def plan_create_packed(mask_bits, row_stride: int, B_Q: int, B_KV: int, N: int, heads: int, d: int, plan_id: int = -1,
                       max_workspace_bytes: int = 0, stream=None, N_kv: int = 0, dtype: str = "bf16",
                       layout: str = "hnd") -> Plan:
    """``bsa_plan_create_packed``: ``mask_bits`` is a uint8 CUDA tensor of bit-packed rows (see ``pack_mask``)."""
    import torch
    assert mask_bits.is_cuda and mask_bits.is_contiguous() and mask_bits.dtype == torch.uint8
    h = ctypes.c_void_p()
    opt = Options(plan_id, DTYPES[dtype], max_workspace_bytes, N_kv, LAYOUTS[layout], 0)
    _check(lib().bsa_plan_create_packed(mask_bits.data_ptr(), row_stride, B_Q, B_KV, N, heads, d, ctypes.byref(opt),
                                        _stream_ptr(stream), ctypes.byref(h)), "bsa_plan_create_packed")
    return Plan(h.value, layout)


class PlanCache:
    """``bsa_plan_cache_*``: prepared plans keyed by a fingerprint of the mask's activity pattern (warm path)."""

    def __init__(self, capacity: int = 64):
        h = ctypes.c_void_p()
        _check(lib().bsa_plan_cache_create(capacity, ctypes.byref(h)), "bsa_plan_cache_create")
        self._h = h.value

    def get(self, mask, B_Q: int, B_KV: int, N: int, heads: int, d: int, plan_id: int = -1, max_workspace_bytes: int = 0,
            stream=None, row_stride: int = 0, N_kv: int = 0, dtype: str = "bf16", layout: str = "hnd"):
        """``bsa_plan_cache_get``: returns ``(plan, hit)``.  ``row_stride`` > 0: ``mask`` is bit-packed (``pack_mask``).
        The plan is shared with the cache; ``plan.destroy()`` only gives it back."""
        import torch
        assert mask.is_cuda and mask.is_contiguous() and mask.dtype in (torch.uint8, torch.bool)
        h = ctypes.c_void_p()
        hit = ctypes.c_int(0)
        opt = Options(plan_id, DTYPES[dtype], max_workspace_bytes, N_kv, LAYOUTS[layout], 0)
        _check(lib().bsa_plan_cache_get(self._h, mask.data_ptr(), row_stride, B_Q, B_KV, N, heads, d, ctypes.byref(opt),
                                        _stream_ptr(stream), ctypes.byref(h), ctypes.byref(hit)), "bsa_plan_cache_get")
        return Plan(h.value, layout), bool(hit.value)

    def request(self, mask, B_Q: int, B_KV: int, N: int, heads: int, d: int, Q, K, V, O, LSE, plan_id: int = -1,
                max_workspace_bytes: int = 0, stream=None, row_stride: int = 0, N_kv: int = 0, dtype: str = "bf16",
                layout: str = "hnd"):
        """``bsa_plan_cache_request``: ``get`` + ``forward`` in one call; returns ``(plan, hit)``."""
        h = ctypes.c_void_p()
        hit = ctypes.c_int(0)
        opt = Options(plan_id, DTYPES[dtype], max_workspace_bytes, N_kv, LAYOUTS[layout], 0)
        _check(lib().bsa_plan_cache_request(self._h, mask.data_ptr(), row_stride, B_Q, B_KV, N, heads, d, Q.data_ptr(),
                                            K.data_ptr(), V.data_ptr(), O.data_ptr(), LSE.data_ptr(), ctypes.byref(opt),
                                            _stream_ptr(stream), ctypes.byref(h), ctypes.byref(hit)),
               "bsa_plan_cache_request")
        return Plan(h.value, layout), bool(hit.value)

    def stats(self) -> Dict:
        a, b, c = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        n = ctypes.c_int32()
        _check(lib().bsa_plan_cache_stats(self._h, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c), ctypes.byref(n)),
               "bsa_plan_cache_stats")
        return {"hits": a.value, "misses": b.value, "evictions": c.value, "entries": n.value}

    def destroy(self):
        if self._h:
            _check(lib().bsa_plan_cache_destroy(self._h), "bsa_plan_cache_destroy")
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def request_host(mask: np.ndarray, B_Q: int, B_KV: int, N: int, heads: int, d: int, Q, K, V, O, LSE,
                 plan_id: int = -1, N_kv: int = 0, dtype: str = "bf16", layout: str = "hnd", batch: int = 0) -> Dict:
    """``bsa_request_host``: all arguments are HOST buffers (torch CPU tensors or numpy arrays)."""
    def ptr(x):
        return x.data_ptr() if hasattr(x, "data_ptr") else x.ctypes.data
    inf = PlanInfo()
    opt = Options(plan_id, DTYPES[dtype], 0, N_kv, LAYOUTS[layout], batch)
    _check(lib().bsa_request_host(ptr(mask), B_Q, B_KV, N, heads, d, ptr(Q), ptr(K), ptr(V), ptr(O), ptr(LSE),
                                  ctypes.byref(opt), ctypes.byref(inf)), "bsa_request_host")
    return inf.as_dict()


# ---------------------------------------------------------------- positions and windows
# The C structs as packed bytes: filling a ctypes structure field by field takes longer than the smallest kernels.
_PTR = struct.Struct("@P")
_VIEW = struct.Struct("@Pqqq")                       # bsa_view_t
_ROPE = struct.Struct("@4iq2i4i4idPPqq4i4i")         # bsa_rope_desc_t
_WINDOW = struct.Struct("@4iqqqqqifPP")              # bsa_window_desc_t
PAIRS = {"interleaved": 0, "halves": 1}  # BSA_PAIRS_*
_PAD = ((0, 0, 0, 0), (0, 0, 0), (0, 0), (0,), ())  # of an array of BSA_MAX_AXES entries behind so many given ones
_torch = None      # the module and its two element types, once a call has needed them
_DTYPE_IDS: Dict = {}


def _tensor_of(t, what: str):
    """(type id, device index) of a call's first tensor."""
    global _torch
    if _torch is None:
        import torch
        _DTYPE_IDS.update({torch.bfloat16: 0, torch.float16: 1})
        _torch = torch
    dt, dev = _DTYPE_IDS.get(t.dtype), t.get_device()
    if dt is None or dev < 0:
        raise ValueError(f"{what} has to be a bf16 or fp16 CUDA tensor")
    return dt, dev


def _view(t, nhd: bool, dtype, dev: int, what: str):
    """(batch, heads, rows, d, packed bsa_view_t) of ``[heads, rows, d]`` / ``[batch, heads, rows, d]``, or of
    ``[rows, heads, d]`` / ``[batch, rows, heads, d]`` with ``nhd``."""
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{what} has to have the type and the device of Q")
    shape = t.shape
    if len(shape) == 4:
        b, h, n, d = shape
        sb, sh, sn, sd = t.stride()
    elif len(shape) == 3:
        b, sb = 1, 0
        h, n, d = shape
        sh, sn, sd = t.stride()
    else:
        raise ValueError(f"{what} has to have three or four dimensions")
    if sd != 1 and d > 1:
        raise ValueError(f"{what} has to be contiguous in its last dimension")
    if nhd:
        return b, n, h, d, _VIEW.pack(t.data_ptr(), sb, sn, sh)
    return b, h, n, d, _VIEW.pack(t.data_ptr(), sb, sh, sn)


def _int32_ptr(t, shapes, dev: int, what: str) -> int:
    if t.dtype is not _torch.int32 or t.get_device() != dev or tuple(t.shape) not in shapes or not t.is_contiguous():
        raise ValueError(f"{what} has to be a contiguous int32 tensor {' or '.join(map(str, shapes))} on the device of Q")
    return t.data_ptr()


def _fresh_view(t, like, nhd: bool, dtype, dev: int, packed: bytes) -> bytes:
    """The view of ``t``, just allocated like ``like``, whose own view is ``packed``: the same strides where ``like`` is dense."""
    if like.is_contiguous():
        return _PTR.pack(t.data_ptr()) + packed[8:]
    return _view(t, nhd, dtype, dev, "out")[4]


def _call(dev: int, stream, where: str, call, *args):
    """``call(*args, stream pointer)`` with device ``dev`` current, on ``stream`` or the device's current stream; raises its errors."""
    if dev != _torch._C._cuda_getDevice():
        with _torch.cuda.device(dev):
            status = call(*args, _stream_ptr(stream))
    else:  # (the handle alone, as in _stream_ptr)
        status = call(*args, (_torch._C._cuda_getCurrentRawStream(dev) or None) if stream is None else _stream_ptr(stream))
    if status:
        _check(status, where)


def rope(Q, K=None, *, axes, positions=None, grid=None, first: int = 0, origin=None, theta: float = 10000.0, freq=None,
         pairs: str = "interleaved", shared_freq: bool = False, inverse: bool = False, layout: str = "hnd", out=None,
         stream=None):
    """``bsa_rope``: rotary positions of Q and, with the same angles, of K.  Returns ``(Q', K')``, or ``Q'`` without K.

    Q, K: bf16 or fp16 CUDA tensors ``[heads, N, d]`` or ``[batch, heads, N, d]`` (``layout="nhd"``: heads behind N), any
    strides that are multiples of 8 elements.  ``axes``: channels that each of the one to four axes rotates.  Either
    ``positions``, int32 ``[N, len(axes)]`` or ``[batch, N, len(axes)]``, or ``grid`` = the axes' lengths: the tokens from
    ``first`` on stand on it row-major, ``origin`` added, and the others stay as they are.  ``freq``: the pairs' own
    frequencies instead of ``theta``'s.  ``inverse=True`` is the way back: gradients, or positions taken off.
    ``out``: the tensors to write (``(Q, K)`` themselves for in place), e.g. views of a cache.
    ``stream``: a torch stream or a handle; fresh outputs come from its pool, as if allocated with it current."""
    nhd = LAYOUTS[layout] == 1
    dt, dev = _tensor_of(Q, "Q")
    dtype = Q.dtype
    b, h, n, d, vq = _view(Q, nhd, dtype, dev, "Q")
    hk, vk, ok, vok = 0, None, None, None
    if K is not None:
        bk, hk, nk, dk, vk = _view(K, nhd, dtype, dev, "K")
        if bk != b or nk != n or dk != d:
            raise ValueError("Q and K have to agree in batch, tokens and channels")
    if out is None:
        if stream is None:
            oq, ok = _torch.empty_like(Q), None if K is None else _torch.empty_like(K)
        else:
            with _pool(stream, dev):
                oq, ok = _torch.empty_like(Q), None if K is None else _torch.empty_like(K)
        voq = _fresh_view(oq, Q, nhd, dtype, dev, vq)
        if K is not None:
            vok = _fresh_view(ok, K, nhd, dtype, dev, vk)
    else:
        oq, ok = (out, None) if K is None else out
        if oq.shape != Q.shape or (K is not None and ok.shape != K.shape):
            raise ValueError("out has to have the shapes of Q and K")
        voq = _view(oq, nhd, dtype, dev, "out")[4]
        if K is not None:
            vok = _view(ok, nhd, dtype, dev, "out")[4]
    na = len(axes)
    if not 1 <= na <= 4 or (positions is None) == (grid is None):
        raise ValueError("one to four axes, and either positions or a grid")
    pad = _PAD[na]
    if grid is not None:
        if len(grid) != na or (origin is not None and len(origin) != na):
            raise ValueError("grid and origin have one entry per axis")
        pos = per_batch = 0
        where = (*grid, *pad, *origin, *pad) if origin is not None else (*grid, *pad, 0, 0, 0, 0)
    else:
        pos = _int32_ptr(positions, ((n, na), (1, n, na), (b, n, na)), dev, "positions")
        per_batch = n * na if positions.dim() == 3 and positions.shape[0] > 1 else 0
        where = (0, 0, 0, 0, 0, 0, 0, 0)
    freqs = None
    if freq is not None:
        if 2 * len(freq) != sum(axes):
            raise ValueError("freq has one entry per pair of channels")
        freqs = (ctypes.c_double * len(freq))(*freq)
    desc = _ROPE.pack(b, h, hk, d, n, dt, na, *axes, *pad, PAIRS[pairs], shared_freq, inverse, 0, theta,
                      0 if freqs is None else ctypes.addressof(freqs), pos, per_batch, first, *where)
    _call(dev, stream, "bsa_rope", lib().bsa_rope, desc, vq, vk, voq, vok)
    return oq if K is None else (oq, ok)


def _window_desc(Q, K, V, left, right, sinks, q_start, kv_len, scale, nhd):
    """(packed bsa_window_desc_t, packed views of Q, K, V, shape of LSE, device): what forward and backward check alike."""
    dt, dev = _tensor_of(Q, "Q")
    dtype = Q.dtype
    b, h, n, d, vq = _view(Q, nhd, dtype, dev, "Q")
    bk, hk, nk, dk, vk = _view(K, nhd, dtype, dev, "K")
    if V.shape != K.shape or bk != b or dk != d or len(Q.shape) != len(K.shape):
        raise ValueError("K and V have to have one shape, and batch and channels of Q")
    vv = _view(V, nhd, dtype, dev, "V")[4]
    desc = _WINDOW.pack(b, h, hk, d, n, nk, left, right, sinks, dt, scale,
                        0 if q_start is None else _int32_ptr(q_start, ((b,),), dev, "q_start"),
                        0 if kv_len is None else _int32_ptr(kv_len, ((b,),), dev, "kv_len"))
    return desc, vq, vk, vv, ((b, h, n) if len(Q.shape) == 4 else (h, n)), dev


def window_forward(Q, K, V, *, left: int, right: int = 0, sinks: int = 0, q_start=None, kv_len=None, scale: float = 0.0,
                   layout: str = "hnd", O=None, LSE=None, stream=None):
    """``bsa_window_forward``: attention of each query to the keys ``p - left .. p + right`` around its position and to the
    first ``sinks`` keys (those up to ``p + right``); -1: no limit on that side.  Returns ``(O, LSE)``.

    Q ``[heads, N, d]`` or ``[batch, heads, N, d]``, K and V likewise with ``heads_kv`` heads and ``N_kv`` tokens
    (``layout="nhd"``: heads behind tokens); any strides that are multiples of 8 elements.  ``q_start``, ``kv_len``: int32
    CUDA tensors ``[batch]``, each sequence's first query position and its number of keys (default: the queries are the last N
    of N_kv positions).  LSE is fp32 ``[batch, heads, N]`` (``[heads, N]``) in either layout.  ``stream``: as for ``rope``."""
    nhd = LAYOUTS[layout] == 1
    desc, vq, vk, vv, shape, dev = _window_desc(Q, K, V, left, right, sinks, q_start, kv_len, scale, nhd)
    if O is not None:
        if O.shape != Q.shape:
            raise ValueError("O has to have the shape of Q")
        vo = _view(O, nhd, Q.dtype, dev, "O")[4]
    if LSE is not None:
        _check_lse(LSE, shape, dev)
    if O is None or LSE is None:
        fresh = O is None
        if stream is None:
            O = _torch.empty_like(Q) if fresh else O
            LSE = Q.new_empty(shape, dtype=_torch.float32) if LSE is None else LSE
        else:
            with _pool(stream, dev):
                O = _torch.empty_like(Q) if fresh else O
                LSE = Q.new_empty(shape, dtype=_torch.float32) if LSE is None else LSE
        if fresh:
            vo = _fresh_view(O, Q, nhd, Q.dtype, dev, vq)
    _call(dev, stream, "bsa_window_forward", lib().bsa_window_forward, desc, vq, vk, vv, vo, LSE.data_ptr())
    return O, LSE


def _check_lse(LSE, shape, dev: int):
    if tuple(LSE.shape) != shape or LSE.dtype is not _torch.float32 or LSE.get_device() != dev or not LSE.is_contiguous():
        raise ValueError(f"LSE has to be a contiguous fp32 tensor {shape} on the device of Q")


def window_backward(Q, K, V, O, LSE, dO, *, left: int, right: int = 0, sinks: int = 0, q_start=None, kv_len=None,
                    scale: float = 0.0, layout: str = "hnd", dQ=None, dK=None, dV=None, stream=None):
    """``bsa_window_backward``: ``(dQ, dK, dV)`` of ``window_forward`` from its inputs, its outputs and the gradient ``dO`` of
    ``O``; arguments as there.  dK and dV are summed over the query heads that share a key head.  The workspace comes from
    torch's allocator, as the outputs do."""
    nhd = LAYOUTS[layout] == 1
    desc, vq, vk, vv, shape, dev = _window_desc(Q, K, V, left, right, sinks, q_start, kv_len, scale, nhd)
    if O.shape != Q.shape or dO.shape != Q.shape:
        raise ValueError("O and dO have to have the shape of Q")
    _check_lse(LSE, shape, dev)
    L = lib()
    if dev != _torch._C._cuda_getDevice():
        with _torch.cuda.device(dev):
            n = L.bsa_window_workspace_bytes(desc)
    else:
        n = L.bsa_window_workspace_bytes(desc)
    # (where the description is refused n is 0, and the call says why)

    def allocate():
        empty = _torch.empty_like
        return (empty(Q) if dQ is None else dQ, empty(K) if dK is None else dK, empty(V) if dV is None else dV,
                _torch.empty(n, dtype=_torch.uint8, device=Q.device))
    if stream is None:
        dQ, dK, dV, ws = allocate()
    else:  # (the workspace's memory is free again when that stream has come past this call)
        with _pool(stream, dev):
            dQ, dK, dV, ws = allocate()
    if dQ.shape != Q.shape or dK.shape != K.shape or dV.shape != K.shape:
        raise ValueError("gradients have to have the shapes of their tensors")
    views = [_view(t, nhd, Q.dtype, dev, n)[4] for t, n in ((O, "O"), (dO, "dO"), (dQ, "dQ"), (dK, "dK"), (dV, "dV"))]
    _call(dev, stream, "bsa_window_backward", L.bsa_window_backward, desc, vq, vk, vv, views[0], LSE.data_ptr(), *views[1:], ws.data_ptr(), n)
    return dQ, dK, dV


def window_status() -> int:
    """``bsa_window_status``: 0, or the status that a windowed kernel on the current device has left since the last look."""
    out = ctypes.c_int(0)
    _check(lib().bsa_window_status(ctypes.byref(out)), "bsa_window_status")
    return out.value


NOALLOC_MAX_ROWS = 1 << 20


def mask_stats_noalloc(mask, out=None, stream=None):
    """``bsa_mask_stats_noalloc``: statistics of a uint8/bool CUDA mask ``[heads, nQb, nKb]`` into an int64
    CUDA tensor of 4 entries, using the library's built-in scratch (no allocation inside the call when
    ``out`` is given; ``stream`` as for ``Plan.forward``).  Returns ``out``; raises ``BsaError`` (UNSUPPORTED) beyond ``NOALLOC_MAX_ROWS`` rows."""
    import torch
    assert mask.is_cuda and mask.is_contiguous() and mask.dtype in (torch.uint8, torch.bool) and mask.dim() == 3
    if out is None:
        with contextlib.nullcontext() if stream is None else _pool(stream, mask.get_device()):
            out = torch.empty(4, dtype=torch.int64, device=mask.device)
    assert out.is_cuda and out.dtype == torch.int64 and out.numel() >= 4 and out.is_contiguous()
    h, nq, nk = mask.shape
    _check(lib().bsa_mask_stats_noalloc(mask.data_ptr(), h, nq, nk, out.data_ptr(), _stream_ptr(stream)),
           "bsa_mask_stats_noalloc")
    return out


def catalog() -> List[Dict]:
    out = []
    for i in range(lib().bsa_catalog_size()):
        d = PlanDesc()
        _check(lib().bsa_catalog_get(i, ctypes.byref(d)), "bsa_catalog_get")
        out.append({f: (getattr(d, f).decode() if f == "name" else getattr(d, f)) for f, _ in PlanDesc._fields_})
    return out


def plan_eligible(plan_id, B_Q, B_KV, N, heads, d, max_workspace_bytes=0, N_kv=0, dtype="bf16") -> bool:
    """``bsa_plan_eligible_ex``: Eligible(P, R) for the request's geometry, token counts, head dim and element type."""
    return bool(lib().bsa_plan_eligible_ex(plan_id, B_Q, B_KV, N, N_kv, heads, d, DTYPES[dtype], max_workspace_bytes))


def debug_set_wait_limit(cycles: int):
    """``bsa_debug_set_wait_limit`` (test hook): limit of the kernels' bounded waits in SM cycles; <= 0 = default."""
    _check(lib().bsa_debug_set_wait_limit(cycles), "bsa_debug_set_wait_limit")


def debug_withhold_arrival(on: bool):
    """``bsa_debug_withhold_arrival`` (test hook): make the next forwards' first V tile never arrive."""
    _check(lib().bsa_debug_withhold_arrival(1 if on else 0), "bsa_debug_withhold_arrival")


def lut_load(path: str):
    _check(lib().bsa_lut_load(path.encode()), "bsa_lut_load")


def lut_clear():
    lib().bsa_lut_clear()


def lut_select(B_Q, B_KV, N, heads, d, density, run_coverage, skew, max_workspace_bytes=0) -> Tuple[int, bool]:
    hit = ctypes.c_int(0)
    pid = lib().bsa_lut_select(B_Q, B_KV, N, heads, d, density, run_coverage, skew, max_workspace_bytes,
                               ctypes.byref(hit))
    return pid, bool(hit.value)


def lut_buckets(N, density, skew, run_coverage) -> List[int]:
    out = (ctypes.c_int32 * 4)()
    lib().bsa_lut_buckets(N, density, skew, run_coverage, out)
    return list(out)


def force_plan(plan_id: int):
    lib().bsa_force_plan(plan_id)


def kernel_launch_count() -> int:
    return int(lib().bsa_kernel_launch_count())
