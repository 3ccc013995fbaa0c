"""Python binding of the CSV-Decode C ABI (include/csv_decode.h) for MI355X.

Argument marshalling only: every step of the path runs in the HIP kernels of libcsvdecode.so.
PyTorch supplies device memory and the stream.  There is no CPU fallback: importing this package
without the built library raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcsvdecode.so")

FLAG_TOPK_CERT, FLAG_SOFTMAX_CERT, FLAG_FALLBACK, FLAG_INVALID_INPUT, FLAG_SOFTMAX_RELAXED, FLAG_ABORTED = 1, 2, 4, 8, 16, 32
SCHEDULE_ROUNDS, SCHEDULE_ALG1 = 0, 1
COMBINE_ALL, COMBINE_ANY = 0, 1
MAX_K, MAX_CLUSTERS, MAX_BATCH = 1024, 8192, 256
F32, BF16 = 0, 1
ACT_BF16, ACT_MX4 = 0, 1
MX4_MAX_BATCH = 65536
LOSS_MAX_ROWS = 4194303

EXPORTS = [
    "csv_build_index", "csv_index_from_arrays", "csv_index_export", "csv_index_dims", "csv_index_free",
    "csv_workspace_create", "csv_workspace_free", "csv_decode_step", "csv_bounds", "csv_full_logits",
    "csv_profile_begin", "csv_profile_end", "csv_last_error", "csv_kmax_init", "csv_kmax_update",
    "csv_workspace_set_spin_limit", "csv_index_use_bf16_centroids",
    "csv_workspace_set_tail_split", "csv_bounds_static", "csv_index_set_bias_table", "csv_index_get_bias_table",
    "csv_index_set_angular", "csv_index_get_angular",
    "csv_mx4_quantize", "csv_mx4_dequantize", "csv_mx4_head_create", "csv_mx4_head_dims", "csv_mx4_head_free",
    "csv_mx4_logits_scratch", "csv_mx4_logits", "csv_token_logprobs_scratch", "csv_token_logprobs",
    "csv_token_logprobs_backward", "csv_policy_loss_scratch", "csv_policy_loss",
]
PROFILE_STAGES = ["bounds", "round0", "tail"]


class BuildOpts(C.Structure):
    _fields_ = [("iters", C.c_int), ("h_init_labels", C.c_void_p), ("h_init_rows", C.c_void_p),
                ("radius_slack", C.c_float), ("centroid_bf16", C.c_int), ("spherical", C.c_int), ("bias_table_m", C.c_int)]


class StepParams(C.Structure):
    _fields_ = [("k", C.c_int), ("eps", C.c_float), ("K_max_rows", C.c_int), ("combine", C.c_int),
                ("max_rounds", C.c_int), ("delta_clusters", C.c_int), ("relax", C.c_int), ("top_p", C.c_float),
                ("schedule", C.c_int)]


class KmaxCtl(C.Structure):
    _fields_ = [("K_max", C.c_double), ("alpha", C.c_double), ("rho_target", C.c_double), ("K_min", C.c_int),
                ("K_cap", C.c_int), ("literal", C.c_int)]


class PolicyParams(C.Structure):
    _fields_ = [("clip_low", C.c_double), ("clip_high", C.c_double), ("beta", C.c_double), ("inv_temperature", C.c_double)]


class StepOut(C.Structure):
    _fields_ = [("d_ids", C.c_void_p), ("d_logits", C.c_void_p), ("d_lse", C.c_void_p), ("d_flags", C.c_void_p),
                ("d_n_rows", C.c_void_p), ("d_n_clusters", C.c_void_p), ("d_rounds", C.c_void_p),
                ("d_sel_clusters", C.c_void_p), ("d_fallback_count", C.c_void_p),
                ("d_probs", C.c_void_p), ("d_cum", C.c_void_p), ("d_nucleus", C.c_void_p)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2511_21702_amd.build` "
                          "(or __graft_entry__.build()) first; there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, ci = C.c_void_p, C.c_int
    lib.csv_last_error.restype = C.c_char_p
    lib.csv_build_index.argtypes = [vp, vp, ci, ci, ci, C.POINTER(BuildOpts), vp, C.POINTER(vp)]
    lib.csv_index_from_arrays.argtypes = [vp, vp, ci, ci, ci, vp, vp, vp, vp, vp, vp, C.POINTER(vp)]
    lib.csv_index_export.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.csv_index_dims.argtypes = [vp, C.POINTER(ci), C.POINTER(ci), C.POINTER(ci)]
    lib.csv_index_free.argtypes = [vp]
    lib.csv_index_free.restype = None
    lib.csv_workspace_create.argtypes = [vp, ci, ci, C.POINTER(vp)]
    lib.csv_workspace_free.argtypes = [vp]
    lib.csv_workspace_free.restype = None
    lib.csv_decode_step.argtypes = [vp, vp, vp, ci, C.POINTER(StepParams), C.POINTER(StepOut), vp]
    lib.csv_bounds.argtypes = [vp, vp, vp, ci, vp, vp, vp]
    lib.csv_full_logits.argtypes = [vp, vp, vp, ci, vp, vp]
    lib.csv_bounds_static.argtypes = [vp, vp, ci, vp, vp, vp]
    lib.csv_index_set_bias_table.argtypes = [vp, ci, vp, vp]
    lib.csv_index_get_bias_table.argtypes = [vp, C.POINTER(ci), vp]
    lib.csv_index_set_angular.argtypes = [vp, vp, vp]
    lib.csv_index_get_angular.argtypes = [vp, C.POINTER(ci), vp]
    lib.csv_profile_begin.argtypes = [vp, ci]
    lib.csv_profile_end.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(ci)]
    lib.csv_kmax_init.argtypes = [C.POINTER(KmaxCtl), ci, ci, ci, C.c_double, C.c_double, ci]
    lib.csv_kmax_update.argtypes = [C.POINTER(KmaxCtl), ci, ci]
    lib.csv_workspace_set_spin_limit.argtypes = [vp, ci]
    lib.csv_index_use_bf16_centroids.argtypes = [vp, vp]
    lib.csv_workspace_set_tail_split.argtypes = [vp, ci]
    i64, sz, cd = C.c_int64, C.c_size_t, C.c_double
    lib.csv_mx4_quantize.argtypes = [vp, ci, i64, ci, ci, vp, vp, vp]
    lib.csv_mx4_dequantize.argtypes = [vp, vp, ci, ci, vp, ci, i64, vp]
    lib.csv_mx4_head_create.argtypes = [vp, vp, vp, ci, ci, vp, C.POINTER(vp)]
    lib.csv_mx4_head_dims.argtypes = [vp, C.POINTER(ci), C.POINTER(ci)]
    lib.csv_mx4_head_free.argtypes = [vp]
    lib.csv_mx4_head_free.restype = None
    lib.csv_mx4_logits_scratch.argtypes = [vp, ci, ci, C.POINTER(sz)]
    lib.csv_mx4_logits.argtypes = [vp, vp, ci, ci, vp, ci, vp, sz, vp]
    lib.csv_token_logprobs_scratch.argtypes = [ci, ci, C.POINTER(sz)]
    lib.csv_policy_loss_scratch.argtypes = [ci, ci, C.POINTER(sz)]
    lib.csv_token_logprobs.argtypes = [vp, ci, i64, ci, ci, vp, cd, vp, vp, vp, sz, vp]
    lib.csv_token_logprobs_backward.argtypes = [vp, ci, i64, ci, ci, vp, vp, vp, cd, vp, i64, vp]
    lib.csv_policy_loss.argtypes = [vp, ci, i64, ci, ci, vp, vp, vp, vp, vp, C.POINTER(PolicyParams), vp, vp, vp, i64, vp, sz, vp]
    return lib


lib = _load()


class CsvError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"csv error {code}: {lib.csv_last_error().decode()}")


def _check(rc: int) -> None:
    if rc != 0:
        raise CsvError(rc)


def _stream(stream=None) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _dev2(t: torch.Tensor, what: str) -> torch.Tensor:
    if not t.is_cuda or t.element_size() != 2 or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous 16-bit (bf16 pattern) CUDA tensor")
    return t


class CsvIndex:
    """Owner of a csv_index handle."""

    def __init__(self, handle: int):
        self._h = C.c_void_p(handle)
        V, d, Cc = C.c_int(), C.c_int(), C.c_int()
        _check(lib.csv_index_dims(self._h, C.byref(V), C.byref(d), C.byref(Cc)))
        self.V, self.d, self.C = V.value, d.value, Cc.value

    def export(self) -> dict:
        import numpy as np
        mu = np.empty((self.C, self.d), np.float32)
        R = np.empty(self.C, np.float32)
        bmax = np.empty(self.C, np.float32)
        n = np.empty(self.C, np.int32)
        perm = np.empty(self.V, np.int32)
        _check(lib.csv_index_export(self._h, mu.ctypes.data, R.ctypes.data, bmax.ctypes.data, n.ctypes.data,
                                    perm.ctypes.data))
        return {"mu": mu, "R": R, "bmax": bmax, "n": n, "perm": perm}

    def set_angular(self, ang, stream=None) -> None:
        """ang: numpy float32 [C, 4] (cos, sin of the angular radius, largest, smallest row norm), or None to remove."""
        import numpy as np
        if ang is None:
            _check(lib.csv_index_set_angular(self._h, None, _stream(stream)))
            return
        t = np.ascontiguousarray(ang, dtype=np.float32)
        assert t.shape == (self.C, 4)
        _check(lib.csv_index_set_angular(self._h, t.ctypes.data, _stream(stream)))

    def angular(self):
        """numpy float32 [C, 4], or None for a Euclidean index."""
        import numpy as np
        present = C.c_int()
        _check(lib.csv_index_get_angular(self._h, C.byref(present), None))
        if not present.value:
            return None
        t = np.empty((self.C, 4), np.float32)
        _check(lib.csv_index_get_angular(self._h, C.byref(present), t.ctypes.data))
        return t

    def set_bias_table(self, table, stream=None) -> None:
        """table: numpy float32 [C, m, 2] of (radius, bias) pairs, or None to remove the table."""
        import numpy as np
        if table is None:
            _check(lib.csv_index_set_bias_table(self._h, 0, None, _stream(stream)))
            return
        t = np.ascontiguousarray(table, dtype=np.float32)
        assert t.ndim == 3 and t.shape[0] == self.C and t.shape[2] == 2
        _check(lib.csv_index_set_bias_table(self._h, t.shape[1], t.ctypes.data, _stream(stream)))

    def bias_table(self):
        """numpy float32 [C, m, 2], or None when the index has no table."""
        import numpy as np
        m = C.c_int()
        _check(lib.csv_index_get_bias_table(self._h, C.byref(m), None))
        if m.value == 0:
            return None
        t = np.empty((self.C, m.value, 2), np.float32)
        _check(lib.csv_index_get_bias_table(self._h, C.byref(m), t.ctypes.data))
        return t

    def free(self) -> None:
        if self._h:
            lib.csv_index_free(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def csv_build_index(W: torch.Tensor, b, C_clusters: int, init_labels=None, init_rows=None, iters: int = 0,
                    radius_slack: float = 2.0 ** -14, stream=None, centroid_bf16: bool = False,
                    bias_table_m: int = 0, spherical: bool = False) -> CsvIndex:
    """W: [V,d] 16-bit CUDA tensor (bf16 patterns, original token order); b: float32 CUDA [V] or None.
    init_labels / init_rows: host int32 numpy arrays (see csv_build_opts)."""
    import numpy as np
    _dev2(W, "W")
    V, d = W.shape
    keep = []
    opts = BuildOpts(iters=iters, h_init_labels=None, h_init_rows=None, radius_slack=radius_slack,
                     centroid_bf16=int(bool(centroid_bf16)), spherical=int(bool(spherical)), bias_table_m=int(bias_table_m))
    if init_labels is not None:
        a = np.ascontiguousarray(init_labels, dtype=np.int32)
        assert a.shape == (V,)
        keep.append(a)
        opts.h_init_labels = a.ctypes.data
    if init_rows is not None:
        a = np.ascontiguousarray(init_rows, dtype=np.int32)
        assert a.shape == (C_clusters,)
        keep.append(a)
        opts.h_init_rows = a.ctypes.data
    out = C.c_void_p()
    bptr = None if b is None else b.data_ptr()
    if b is not None:
        assert b.is_cuda and b.dtype == torch.float32 and b.is_contiguous() and b.numel() == V
    _check(lib.csv_build_index(W.data_ptr(), bptr, V, d, C_clusters, C.byref(opts), _stream(stream), C.byref(out)))
    return CsvIndex(out.value)


def csv_index_from_arrays(W: torch.Tensor, b, mu, R, bmax, n, perm, stream=None, centroid_bf16: bool = False) -> CsvIndex:
    """Import metadata computed elsewhere (host numpy arrays).  centroid_bf16: mu holds bfloat16 values (and the
    radii were measured to them); the index then keeps and reads the centroids as bfloat16."""
    import numpy as np
    _dev2(W, "W")
    V, d = W.shape
    mu = np.ascontiguousarray(mu, dtype=np.float32)
    R = np.ascontiguousarray(R, dtype=np.float32)
    bmax = np.ascontiguousarray(bmax, dtype=np.float32)
    n = np.ascontiguousarray(n, dtype=np.int32)
    perm = np.ascontiguousarray(perm, dtype=np.int32)
    Cc = mu.shape[0]
    assert mu.shape == (Cc, d) and R.shape == (Cc,) and bmax.shape == (Cc,) and n.shape == (Cc,) and perm.shape == (V,)
    out = C.c_void_p()
    bptr = None if b is None else b.data_ptr()
    _check(lib.csv_index_from_arrays(W.data_ptr(), bptr, V, d, Cc, mu.ctypes.data, R.ctypes.data, bmax.ctypes.data,
                                     n.ctypes.data, perm.ctypes.data, _stream(stream), C.byref(out)))
    idx = CsvIndex(out.value)
    if centroid_bf16:
        _check(lib.csv_index_use_bf16_centroids(idx._h, _stream(stream)))
    return idx


class CsvWorkspace:
    def __init__(self, index: CsvIndex, B_max: int, K_cap_rows: int):
        out = C.c_void_p()
        _check(lib.csv_workspace_create(index._h, B_max, K_cap_rows, C.byref(out)))
        self._h = out
        self.index = index
        self.B_max, self.K_cap = B_max, K_cap_rows

    def set_tail_split(self, min_batch: int) -> None:
        """Batches of at least min_batch sequences run the tail as one launch per phase (0 = follow recent steps)."""
        _check(lib.csv_workspace_set_tail_split(self._h, min_batch))

    def set_spin_limit(self, polls: int) -> None:
        """Polls a grid barrier of the tail kernel waits before giving the step up (0 = default)."""
        _check(lib.csv_workspace_set_spin_limit(self._h, polls))

    def profile_begin(self, max_steps: int) -> None:
        _check(lib.csv_profile_begin(self._h, max_steps))

    def profile_end(self) -> tuple[dict, int]:
        """(summed milliseconds per stage, recorded steps)."""
        ms = (C.c_float * len(PROFILE_STAGES))()
        n = C.c_int()
        _check(lib.csv_profile_end(self._h, ms, C.byref(n)))
        return dict(zip(PROFILE_STAGES, list(ms))), n.value

    def free(self) -> None:
        if self._h:
            lib.csv_workspace_free(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


@dataclass
class StepBuffers:
    """Device output buffers of csv_decode_step plus the ctypes structs that point at them."""
    ids: torch.Tensor
    logits: torch.Tensor
    lse: torch.Tensor
    flags: torch.Tensor
    n_rows: torch.Tensor
    n_clusters: torch.Tensor
    rounds: torch.Tensor
    sel_clusters: torch.Tensor | None
    fallback_count: torch.Tensor
    params: StepParams
    out: StepOut
    probs: torch.Tensor | None = None
    cum: torch.Tensor | None = None
    nucleus: torch.Tensor | None = None


def make_step_buffers(index: CsvIndex, B: int, k: int, eps: float, K_max_rows: int, combine: int = COMBINE_ALL,
                      want_sel: bool = False, device="cuda", max_rounds: int = 0, delta_clusters: int = 0,
                      relax: bool = False, want_dist: bool = False, top_p: float = 0.0, schedule: int = 0) -> StepBuffers:
    kk = max(k, 1)
    ids = torch.full((B, kk), -2, dtype=torch.int32, device=device)
    logits = torch.zeros((B, kk), dtype=torch.float32, device=device)
    lse = torch.zeros(B, dtype=torch.float32, device=device)
    flags = torch.zeros(B, dtype=torch.int32, device=device)
    n_rows = torch.zeros(B, dtype=torch.int32, device=device)
    n_clusters = torch.zeros(B, dtype=torch.int32, device=device)
    rounds = torch.zeros(B, dtype=torch.int32, device=device)
    sel = torch.full((B, index.C), -1, dtype=torch.int32, device=device) if want_sel else None
    fbc = torch.zeros(1, dtype=torch.int64, device=device)
    probs = torch.full((B, kk), -1.0, dtype=torch.float32, device=device) if want_dist else None
    cum = torch.full((B, kk), -1.0, dtype=torch.float32, device=device) if want_dist else None
    nucleus = torch.full((B,), -1, dtype=torch.int32, device=device) if want_dist else None
    params = StepParams(k=k, eps=eps, K_max_rows=K_max_rows, combine=combine, max_rounds=max_rounds,
                        delta_clusters=delta_clusters, relax=int(bool(relax)), top_p=top_p, schedule=schedule)
    out = StepOut(ids.data_ptr(), logits.data_ptr(), lse.data_ptr(), flags.data_ptr(), n_rows.data_ptr(),
                  n_clusters.data_ptr(), rounds.data_ptr(), sel.data_ptr() if want_sel else None, fbc.data_ptr(),
                  probs.data_ptr() if want_dist else None, cum.data_ptr() if want_dist else None,
                  nucleus.data_ptr() if want_dist else None)
    return StepBuffers(ids, logits, lse, flags, n_rows, n_clusters, rounds, sel, fbc, params, out, probs, cum, nucleus)


def csv_decode_step(ws: CsvWorkspace, index: CsvIndex, h: torch.Tensor, buf: StepBuffers, stream=None) -> StepBuffers:
    """Enqueue one certified decode step for h [B,d] (bf16 patterns).  Results land in `buf` after a stream sync."""
    _dev2(h, "h")
    B = h.shape[0]
    _check(lib.csv_decode_step(ws._h, index._h, h.data_ptr(), B, C.byref(buf.params), C.byref(buf.out), _stream(stream)))
    return buf


def csv_decode_step_raw(ws: CsvWorkspace, index: CsvIndex, h_ptr: int, B: int, buf: StepBuffers, stream_ptr: int) -> None:
    """Same call with a raw device pointer and stream handle (tight loops: no tensor checks)."""
    rc = lib.csv_decode_step(ws._h, index._h, h_ptr, B, C.byref(buf.params), C.byref(buf.out), stream_ptr)
    if rc:
        raise CsvError(rc)


def csv_bounds(ws: CsvWorkspace, index: CsvIndex, h: torch.Tensor, stream=None):
    _dev2(h, "h")
    B = h.shape[0]
    U = torch.empty((B, index.C), dtype=torch.float32, device=h.device)
    hn = torch.empty(B, dtype=torch.float32, device=h.device)
    _check(lib.csv_bounds(ws._h, index._h, h.data_ptr(), B, U.data_ptr(), hn.data_ptr(), _stream(stream)))
    return U, hn


def csv_bounds_static(index: CsvIndex, h: torch.Tensor, U: torch.Tensor, hn: torch.Tensor, stream=None) -> None:
    """csv_bounds without a workspace and without any allocation: the caller passes the output tensors
    U [B,C] float32 and hn [B] float32."""
    _dev2(h, "h")
    B = h.shape[0]
    assert U.is_cuda and U.dtype == torch.float32 and U.is_contiguous() and tuple(U.shape) == (B, index.C)
    assert hn.is_cuda and hn.dtype == torch.float32 and hn.is_contiguous() and hn.numel() == B
    _check(lib.csv_bounds_static(index._h, h.data_ptr(), B, U.data_ptr(), hn.data_ptr(), _stream(stream)))


def csv_full_logits(ws: CsvWorkspace, index: CsvIndex, h: torch.Tensor, out: torch.Tensor | None = None, stream=None):
    _dev2(h, "h")
    B = h.shape[0]
    if out is None:
        out = torch.empty((B, index.V), dtype=torch.float32, device=h.device)
    _check(lib.csv_full_logits(ws._h, index._h, h.data_ptr(), B, out.data_ptr(), _stream(stream)))
    return out


_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.int16: BF16}     # int16: bf16 patterns

# The calls below are short next to a kernel of a few microseconds, so their checks are plain comparisons; the device and the raw stream
# are asked for without building stream objects.
_current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _rows(t: torch.Tensor, what: str) -> tuple:
    """(element type, device, elements from row to row) of a [rows, columns] tensor on the current device whose rows are contiguous."""
    ty, dev = _TYPES.get(t.dtype), t.get_device()
    if ty is None or t.dim() != 2:
        raise ValueError(f"{what} must be 2-D, float32 or bfloat16")
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{what} must have contiguous rows")
    if dev < 0 or dev != _current_device():
        raise ValueError(f"{what} must be on the current CUDA device")
    return ty, dev, ld if rows > 1 else cols


def _dense(t: torch.Tensor, what: str, dtype, shape: tuple, dev: int) -> int:
    """Pointer of a contiguous tensor of this type and shape on device `dev`."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {shape} on the device of the call")
    return t.data_ptr()


def _vector(t: torch.Tensor, what: str, dtype, n: int, dev: int) -> int:
    """Pointer of a contiguous tensor of this type with n elements on device `dev`."""
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of {n} elements on the device of the call")
    return t.data_ptr()


def _device_of(t: torch.Tensor, what: str) -> int:
    dev = t.get_device()
    if dev < 0 or dev != _current_device():
        raise ValueError(f"{what} must be on the current CUDA device")
    return dev


def _scratch(need: int, scratch, dev: int) -> tuple:
    """(tensor that keeps the memory alive, pointer, bytes); the caller's scratch where it is given."""
    if scratch is not None:
        if scratch.get_device() != dev or not scratch.is_contiguous():
            raise ValueError("scratch must be contiguous and on the device of the call")
        return scratch, scratch.data_ptr(), scratch.numel() * scratch.element_size()
    if need == 0:
        return None, None, 0
    t = torch.empty(need, dtype=torch.uint8, device=dev)
    return t, t.data_ptr(), need


def mx4_padded(d: int) -> int:
    """Elements of a 4-bit row with its padding: two per byte of codes, 32 per scale byte."""
    return (d + 127) // 128 * 128


def csv_mx4_quantize(x: torch.Tensor, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None, stream=None):
    """(codes uint8 [rows, dp/2], scales uint8 [rows, dp/32]) of the rows of x, bfloat16 or float32 [rows, d]."""
    if stream is not None:
        with torch.cuda.stream(stream):         # what the call allocates belongs to the stream that it runs on
            return csv_mx4_quantize(x, codes, scales)
    ty, dev, ld = _rows(x, "x")
    rows, d = x.shape
    dp = mx4_padded(d)
    if codes is None:
        codes = torch.empty((rows, dp // 2), dtype=torch.uint8, device=dev)
    if scales is None:
        scales = torch.empty((rows, dp // 32), dtype=torch.uint8, device=dev)
    _check(lib.csv_mx4_quantize(x.data_ptr(), ty, ld, rows, d, _dense(codes, "codes", torch.uint8, (rows, dp // 2), dev),
                                _dense(scales, "scales", torch.uint8, (rows, dp // 32), dev), _raw_stream(dev)))
    return codes, scales


def csv_mx4_dequantize(codes: torch.Tensor, scales: torch.Tensor, d: int, out: torch.Tensor | None = None, dtype=torch.bfloat16, stream=None):
    """The values [rows, d] that codes and scales stand for."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return csv_mx4_dequantize(codes, scales, d, out, dtype)
    rows, dp = codes.shape[0], mx4_padded(d)
    if out is None:
        out = torch.empty((rows, d), dtype=dtype, device=_device_of(codes, "codes"))
    ty, dev, ld = _rows(out, "out")
    if out.shape != (rows, d):
        raise ValueError(f"out must have the shape {(rows, d)}")
    _check(lib.csv_mx4_dequantize(_dense(codes, "codes", torch.uint8, (rows, dp // 2), dev), _dense(scales, "scales", torch.uint8, (rows, dp // 32), dev),
                                  rows, d, out.data_ptr(), ty, ld, _raw_stream(dev)))
    return out


class CsvMx4Head:
    """Owner of a csv_mx4_head handle."""

    def __init__(self, handle: int):
        self._h = C.c_void_p(handle)
        V, d = C.c_int(), C.c_int()
        _check(lib.csv_mx4_head_dims(self._h, C.byref(V), C.byref(d)))
        self.V, self.d = V.value, d.value

    def scratch_bytes(self, B: int, act: int) -> int:
        """Bytes of scratch that csv_mx4_logits needs for B hidden states."""
        need = C.c_size_t()
        _check(lib.csv_mx4_logits_scratch(self._h, B, act, C.byref(need)))
        return need.value

    def free(self) -> None:
        if self._h:
            lib.csv_mx4_head_free(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def csv_mx4_head(codes: torch.Tensor, scales: torch.Tensor, b, d: int, stream=None) -> CsvMx4Head:
    """A head of 4-bit rows [V, d] (csv_mx4_quantize of W, or a checkpoint), laid out for csv_mx4_logits; b: float32 CUDA [V] or None."""
    V, dp, dev = codes.shape[0], mx4_padded(d), _device_of(codes, "codes")
    out = C.c_void_p()
    _check(lib.csv_mx4_head_create(_dense(codes, "codes", torch.uint8, (V, dp // 2), dev), _dense(scales, "scales", torch.uint8, (V, dp // 32), dev),
                                   None if b is None else _dense(b, "b", torch.float32, (V,), dev), V, d, _stream(stream), C.byref(out)))
    return CsvMx4Head(out.value)


def csv_mx4_logits(head: CsvMx4Head, h: torch.Tensor, out: torch.Tensor | None = None, act: int = ACT_BF16, dtype=torch.float32,
                   scratch: torch.Tensor | None = None, stream=None):
    """Logits [B, V] of hidden states h [B, d] (bf16 patterns) from a 4-bit head; act ACT_MX4 rounds h to 4 bits first."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return csv_mx4_logits(head, h, out, act, dtype, scratch)
    dev = _device_of(h, "h")
    if h.dim() != 2 or h.shape[1] != head.d or h.dtype not in (torch.bfloat16, torch.int16) or not h.is_contiguous():
        raise ValueError(f"h must be a contiguous [B, {head.d}] tensor in bfloat16")
    B = h.shape[0]
    if out is None:
        out = torch.empty((B, head.V), dtype=dtype, device=dev)
    ty = _TYPES.get(out.dtype)
    if ty is None:
        raise ValueError("out must be float32 or bfloat16")
    keep, ptr, size = _scratch(0 if act == ACT_BF16 else head.scratch_bytes(B, act), scratch, dev)
    _check(lib.csv_mx4_logits(head._h, h.data_ptr(), B, act, _dense(out, "out", out.dtype, (B, head.V), dev), ty, ptr, size,
                              _raw_stream(dev)))
    return out


@functools.lru_cache(maxsize=256)
def csv_token_logprobs_scratch(N: int, V: int) -> int:
    """Bytes of scratch that csv_token_logprobs needs for logits [N, V]."""
    need = C.c_size_t()
    _check(lib.csv_token_logprobs_scratch(N, V, C.byref(need)))
    return need.value


@functools.lru_cache(maxsize=256)
def csv_policy_loss_scratch(N: int, V: int) -> int:
    """Bytes of scratch that csv_policy_loss needs for logits [N, V]."""
    need = C.c_size_t()
    _check(lib.csv_policy_loss_scratch(N, V, C.byref(need)))
    return need.value


def csv_token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, inv_temperature: float = 1.0, logp: torch.Tensor | None = None,
                       stats: torch.Tensor | None = None, scratch: torch.Tensor | None = None, stream=None):
    """(logp float32 [N], stats float32 [N, 2]) of tokens int32 [N] under logits [N, V], float32 or bfloat16."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return csv_token_logprobs(logits, tokens, inv_temperature, logp, stats, scratch)
    ty, dev, ld = _rows(logits, "logits")
    N, V = logits.shape
    if logp is None:
        logp = torch.empty(N, dtype=torch.float32, device=dev)
    if stats is None:
        stats = torch.empty((N, 2), dtype=torch.float32, device=dev)
    keep, ptr, size = _scratch(csv_token_logprobs_scratch(N, V), scratch, dev)
    _check(lib.csv_token_logprobs(logits.data_ptr(), ty, ld, N, V, _vector(tokens, "tokens", torch.int32, N, dev), inv_temperature,
                                  _vector(logp, "logp", torch.float32, N, dev), _vector(stats, "stats", torch.float32, 2 * N, dev), ptr, size,
                                  _raw_stream(dev)))
    return logp, stats


def _grad_of(logits: torch.Tensor, grad: torch.Tensor, ty: int, dev: int) -> tuple:
    gty, gdev, gld = _rows(grad, "grad")
    if gty != ty or gdev != dev or grad.shape != logits.shape:
        raise ValueError("grad must have the type, the shape and the device of the logits")
    return grad.data_ptr(), gld


def csv_token_logprobs_backward(logits: torch.Tensor, tokens: torch.Tensor, stats: torch.Tensor, grad_logp: torch.Tensor,
                                inv_temperature: float = 1.0, grad: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The gradient by the logits, [N, V] in their type, from the stats of csv_token_logprobs and the gradient by logp (float32 [N]).
    grad may be the logits themselves."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return csv_token_logprobs_backward(logits, tokens, stats, grad_logp, inv_temperature, grad)
    ty, dev, ld = _rows(logits, "logits")
    N, V = logits.shape
    if grad is None:
        grad = torch.empty((N, V), dtype=logits.dtype, device=dev)
    gp, gld = _grad_of(logits, grad, ty, dev)
    _check(lib.csv_token_logprobs_backward(logits.data_ptr(), ty, ld, N, V, _vector(tokens, "tokens", torch.int32, N, dev),
                                           _vector(stats, "stats", torch.float32, 2 * N, dev), _vector(grad_logp, "grad_logp", torch.float32, N, dev),
                                           inv_temperature, gp, gld, _raw_stream(dev)))
    return grad


def csv_policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor, ref_logp: torch.Tensor | None, advantages: torch.Tensor,
                    weights: torch.Tensor, clip_low: float = 0.2, clip_high: float = 0.2, beta: float = 0.0, inv_temperature: float = 1.0,
                    loss: torch.Tensor | None = None, logp: torch.Tensor | None = None, grad: torch.Tensor | None = None, want_grad: bool = True,
                    scratch: torch.Tensor | None = None, stream=None):
    """(loss float32 scalar tensor, logp float32 [N], grad [N, V] in the type of the logits, or None without want_grad and grad) of the
    clipped policy loss; weights are mask and normaliser in one.  grad may be the logits themselves; no other output may share memory with an input.
    Rows that a mask leaves nothing of add 0; a masked token has ratio 0."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return csv_policy_loss(logits, tokens, old_logp, ref_logp, advantages, weights, clip_low, clip_high, beta, inv_temperature, loss,
                                   logp, grad, want_grad, scratch)
    ty, dev, ld = _rows(logits, "logits")
    N, V = logits.shape
    f32 = torch.float32
    if loss is None:
        loss = torch.empty((), dtype=f32, device=dev)
    if logp is None:
        logp = torch.empty(N, dtype=f32, device=dev)
    if grad is None and want_grad:
        grad = torch.empty((N, V), dtype=logits.dtype, device=dev)
    gp, gld = (None, 0) if grad is None else _grad_of(logits, grad, ty, dev)
    keep, ptr, size = _scratch(csv_policy_loss_scratch(N, V), scratch, dev)
    _check(lib.csv_policy_loss(logits.data_ptr(), ty, ld, N, V, _vector(tokens, "tokens", torch.int32, N, dev), _vector(old_logp, "old_logp", f32, N, dev),
                               None if ref_logp is None else _vector(ref_logp, "ref_logp", f32, N, dev), _vector(advantages, "advantages", f32, N, dev),
                               _vector(weights, "weights", f32, N, dev), C.byref(PolicyParams(clip_low, clip_high, beta, inv_temperature)),
                               _vector(loss, "loss", f32, 1, dev), _vector(logp, "logp", f32, N, dev), gp, gld, ptr, size,
                               _raw_stream(dev)))
    return loss, logp, grad


def bits_to_device(bits) -> torch.Tensor:
    """numpy uint16 bf16 patterns -> CUDA int16 tensor with the same bits."""
    import numpy as np
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda()


class KmaxController:
    """Host-side adaptive row budget (csv_kmax_init / csv_kmax_update)."""

    def __init__(self, K0: int, K_min: int, K_cap: int, alpha: float = 0.01, rho_target: float = 0.02, literal: bool = False):
        self.ctl = KmaxCtl()
        _check(lib.csv_kmax_init(C.byref(self.ctl), K0, K_min, K_cap, alpha, rho_target, int(literal)))

    def update(self, n_fallback: int, n_sequences: int) -> int:
        rc = lib.csv_kmax_update(C.byref(self.ctl), n_fallback, n_sequences)
        if rc < 0:
            raise CsvError(rc)
        return rc

    @property
    def value(self) -> float:
        return self.ctl.K_max
