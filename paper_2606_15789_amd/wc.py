"""Python binding of libwc (ctypes): argument marshalling only.

Every step of the decode runs in libwc's HIP kernel; this module converts
numpy / torch objects to the plain pointers and sizes of the C ABI declared in
``include/wc.h`` and raises on any non-zero status.  There is no fallback: if
``libwc.so`` is missing or fails to load, every call raises.
"""

from __future__ import annotations

import contextlib
import ctypes as C
import operator
import os
import struct
from collections import namedtuple

import numpy as np

from . import build as _build

DTYPES = {"bf16": 1, "fp16": 2, "u8": 3, "u4": 4, "fp8_e4m3": 5, "fp8_e5m2": 6, "fp4_e2m1": 7}
_DTYPE_NAMES = {v: k for k, v in DTYPES.items()}
STATUS = {0: "WC_OK", -1: "WC_EINVAL", -2: "WC_ENOMEM", -3: "WC_ECORRUPT", -4: "WC_EHIP",
          -5: "WC_EUNSUPPORTED"}
DERR = {1: "WC_DERR_INDEX", 2: "WC_DERR_STATE", 4: "WC_DERR_CURSOR", 8: "WC_DERR_TABLE"}

# Every function the header declares; the library must export all of them.
EXPORTS = ["wc_analyze", "wc_encode", "wc_open", "wc_decode", "wc_gemv", "wc_free",
           "wc_version", "wc_analyze_device", "wc_encode_device_bounds", "wc_encode_device",
           "wc_gemm_workspace_bytes", "wc_gemm", "wc_gemm_i8", "wc_gemv_mx", "wc_gemv_w4",
           "wc_stream", "wc_analyze_device_static", "wc_quantize_i8",
           "wc_matmul_i8_workspace_bytes", "wc_matmul_i8", "wc_linear_i8_workspace_bytes",
           "wc_linear_i8", "wc_route_workspace_bytes", "wc_route",
           "wc_experts_i8_workspace_bytes", "wc_experts_i8"]

ANALYZE_WORKSPACE_BYTES = 524288  # WC_ANALYZE_WORKSPACE_BYTES


class WcError(RuntimeError):
    def __init__(self, what, rc):
        super().__init__(f"{what} failed: {STATUS.get(rc, rc)}")
        self.rc = rc


class _Tensor(C.Structure):
    _fields_ = [("host_ptr", C.c_void_p), ("nbytes", C.c_uint64), ("dtype", C.c_int32),
                ("reserved", C.c_int32), ("rows", C.c_uint64), ("cols", C.c_uint64)]


class _Params(C.Structure):
    _fields_ = [("chunk_bytes", C.c_uint32), ("lanes", C.c_uint32), ("prob_bits", C.c_uint32),
                ("n_threads", C.c_uint32), ("tile_rows", C.c_uint32), ("tile_cols", C.c_uint32),
                ("codebook", C.c_uint32), ("tile_order", C.c_uint32)]


CODEBOOKS = {"tensor": 0, "layer": 1}


class _Stats(C.Structure):
    _fields_ = [("n_fields", C.c_uint32), ("alphabet", C.c_uint32 * 2),
                ("count", C.c_uint64 * 2), ("hist", (C.c_uint64 * 256) * 2),
                ("H", C.c_double * 2), ("H_joint16", C.c_double),
                ("bound_bytes", C.c_double), ("bound_bytes_raw8", C.c_double)]


class _Blob(C.Structure):
    _fields_ = [("data", C.POINTER(C.c_uint8)), ("size", C.c_uint64),
                ("n_tensors", C.c_uint32), ("reserved", C.c_uint32),
                ("n_chunks", C.c_uint64), ("out_bytes", C.POINTER(C.c_uint64)),
                ("meta_bytes", C.c_uint64), ("record_hdr_bytes", C.c_uint64),
                ("state_bytes", C.c_uint64), ("word_bytes", C.c_uint64),
                ("pad_bytes", C.c_uint64), ("raw_bytes", C.c_uint64),
                ("priv", C.c_void_p)]


class _I8Job(C.Structure):
    _fields_ = [("w", C.c_void_p), ("scale", C.c_void_p), ("bias", C.c_void_p),
                ("y", C.c_void_p), ("ldw", C.c_uint64), ("ldy", C.c_uint64), ("n", C.c_uint32),
                ("scale_dtype", C.c_int32), ("bias_dtype", C.c_int32), ("y_dtype", C.c_int32)]


class _RouteParams(C.Structure):
    _fields_ = [("experts", C.c_uint32), ("k", C.c_uint32), ("score", C.c_int32),
                ("renormalize", C.c_int32), ("groups", C.c_uint32), ("top_groups", C.c_uint32),
                ("group_top", C.c_uint32), ("scale", C.c_float)]


class _I8Experts(C.Structure):
    _fields_ = [("w", C.c_void_p), ("scale", C.c_void_p), ("stride", C.c_uint64),
                ("scale_dtype", C.c_int32), ("reserved", C.c_int32)]


_lib = None


def lib():
    """Load libwc.so (building it first only if nothing is built)."""
    global _lib
    if _lib is None:
        # WC_LIB selects another build of libwc (for A/B measurements of kernel variants)
        path = os.environ.get("WC_LIB") or _build.ensure_built()
        L = C.CDLL(path)
        L.wc_analyze.argtypes = [C.POINTER(_Tensor), C.POINTER(_Stats)]
        L.wc_analyze.restype = C.c_int
        L.wc_encode.argtypes = [C.POINTER(_Tensor), C.c_uint32, C.POINTER(_Params),
                                C.POINTER(C.POINTER(_Blob))]
        L.wc_encode.restype = C.c_int
        L.wc_open.argtypes = [C.c_void_p, C.c_uint64, C.POINTER(C.POINTER(_Blob))]
        L.wc_open.restype = C.c_int
        L.wc_decode.argtypes = [C.POINTER(_Blob), C.c_void_p, C.POINTER(C.c_void_p), C.c_uint32,
                                C.c_void_p, C.c_void_p]
        L.wc_decode.restype = C.c_int
        L.wc_gemv.argtypes = [C.POINTER(_Blob), C.c_void_p, C.c_uint32,
                              C.POINTER(C.c_uint32), C.POINTER(C.c_void_p), C.c_uint32,
                              C.POINTER(C.c_void_p), C.c_void_p, C.c_void_p]
        L.wc_gemv.restype = C.c_int
        L.wc_gemm_workspace_bytes.argtypes = [C.POINTER(_Blob), C.c_uint32,
                                              C.POINTER(C.c_uint32), C.POINTER(C.c_void_p),
                                              C.c_uint32, C.POINTER(C.c_uint64)]
        L.wc_gemm_workspace_bytes.restype = C.c_int
        L.wc_gemm.argtypes = [C.POINTER(_Blob), C.c_void_p, C.c_uint32, C.POINTER(C.c_uint32),
                              C.POINTER(C.c_void_p), C.c_uint32, C.POINTER(C.c_void_p),
                              C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]
        L.wc_gemm.restype = C.c_int
        L.wc_gemm_i8.argtypes = [C.POINTER(_Blob), C.c_void_p, C.c_uint32, C.POINTER(C.c_uint32),
                                 C.POINTER(C.c_void_p), C.c_uint32, C.POINTER(C.c_void_p),
                                 C.c_void_p, C.c_void_p]
        L.wc_gemm_i8.restype = C.c_int
        L.wc_gemv_mx.argtypes = [C.POINTER(_Blob), C.c_void_p, C.c_uint32, C.POINTER(C.c_uint32),
                                 C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_uint32,
                                 C.POINTER(C.c_void_p), C.c_void_p, C.c_void_p]
        L.wc_gemv_mx.restype = C.c_int
        L.wc_gemv_w4.argtypes = [C.POINTER(_Blob), C.c_void_p, C.c_uint32, C.POINTER(C.c_uint32),
                                 C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                 C.POINTER(C.c_void_p), C.c_uint32, C.POINTER(C.c_void_p),
                                 C.c_void_p, C.c_void_p]
        L.wc_gemv_w4.restype = C.c_int
        L.wc_analyze_device.argtypes = [C.POINTER(_Tensor), C.c_void_p, C.c_uint64, C.c_void_p,
                                        C.POINTER(_Stats)]
        L.wc_analyze_device.restype = C.c_int
        L.wc_analyze_device_static.argtypes = [C.POINTER(_Tensor), C.c_void_p, C.POINTER(_Stats)]
        L.wc_analyze_device_static.restype = C.c_int
        L.wc_encode_device_bounds.argtypes = [C.POINTER(_Tensor), C.c_uint32, C.POINTER(_Params),
                                              C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
        L.wc_encode_device_bounds.restype = C.c_int
        L.wc_encode_device.argtypes = [C.POINTER(_Tensor), C.c_uint32, C.POINTER(_Params),
                                       C.c_void_p, C.c_uint64, C.c_void_p, C.c_uint64,
                                       C.c_void_p, C.c_void_p]
        L.wc_encode_device.restype = C.c_int
        L.wc_stream.argtypes = [C.c_void_p, C.c_uint64, C.c_void_p, C.c_uint64, C.c_uint32,
                                C.c_void_p, C.POINTER(C.c_uint64)]
        L.wc_stream.restype = C.c_int
        job = C.c_void_p  # wc_i8_job array: packed bytes or a ctypes array
        experts = C.POINTER(_I8Experts)
        L.wc_quantize_i8.argtypes = [C.c_void_p, C.c_int32, C.c_uint32, C.c_uint32, C.c_uint64,
                                     C.c_void_p, C.c_void_p, C.c_void_p]
        L.wc_matmul_i8_workspace_bytes.argtypes = [C.c_uint32, C.c_uint32, C.c_uint32, job,
                                                   C.POINTER(C.c_uint64)]
        L.wc_matmul_i8.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint32, C.c_uint32, job,
                                   C.c_void_p, C.c_uint64, C.c_void_p]
        L.wc_linear_i8_workspace_bytes.argtypes = L.wc_matmul_i8_workspace_bytes.argtypes
        L.wc_linear_i8.argtypes = [C.c_void_p, C.c_int32, C.c_uint32, C.c_uint32, C.c_uint64,
                                   C.c_uint32, job, C.c_void_p, C.c_uint64, C.c_void_p]
        L.wc_route_workspace_bytes.argtypes = [C.c_uint32, C.POINTER(_RouteParams),
                                               C.POINTER(C.c_uint64)]
        L.wc_route.argtypes = [C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64,
                               C.POINTER(_RouteParams)] + [C.c_void_p] * 6 + [C.c_uint64,
                                                                              C.c_void_p]
        L.wc_experts_i8_workspace_bytes.argtypes = [C.c_uint32] * 5 + [C.POINTER(C.c_uint64)]
        L.wc_experts_i8.argtypes = [C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64] \
            + [C.c_uint32] * 4 + [C.c_void_p] * 4 + [experts] * 3 \
            + [C.c_void_p, C.c_uint64, C.c_void_p, C.c_uint64, C.c_void_p]
        for name in EXPORTS[EXPORTS.index("wc_quantize_i8"):]:
            getattr(L, name).restype = C.c_int
        L.wc_free.argtypes = [C.POINTER(_Blob)]
        L.wc_free.restype = None
        L.wc_version.restype = C.c_int32
        _lib = L
    return _lib


def library_path() -> str:
    return os.environ.get("WC_LIB") or _build.LIB


def _bytes(data) -> np.ndarray:
    a = np.ascontiguousarray(data)
    return a.view(np.uint8).reshape(-1)


def analyze(dtype: str, data) -> dict:
    """wc_analyze: per-field histograms and empirical entropy of one tensor."""
    b = _bytes(data)
    t = _Tensor(b.ctypes.data if b.size else None, b.size, DTYPES[dtype], 0, 0, 0)
    st = _Stats()
    rc = lib().wc_analyze(C.byref(t), C.byref(st))
    if rc:
        raise WcError("wc_analyze", rc)
    return _stats_dict(st)


def _stats_dict(st) -> dict:
    nf = st.n_fields
    return {"n_fields": nf, "alphabet": [st.alphabet[i] for i in range(nf)],
            "count": [st.count[i] for i in range(nf)],
            "hist": [np.array(st.hist[i][:st.alphabet[i]], np.uint64) for i in range(nf)],
            "H": [st.H[i] for i in range(nf)], "H_joint16": st.H_joint16,
            "bound_bytes": st.bound_bytes, "bound_bytes_raw8": st.bound_bytes_raw8}


class Blob:
    """Owner of a wc_blob (released with wc_free)."""

    def __init__(self, ptr):
        self._p = ptr
        b = ptr.contents
        self.size = int(b.size)
        self.n_tensors = int(b.n_tensors)
        self.n_chunks = int(b.n_chunks)
        self.out_bytes = [int(b.out_bytes[i]) for i in range(self.n_tensors)]
        self.breakdown = {k: int(getattr(b, k)) for k in
                          ("meta_bytes", "record_hdr_bytes", "state_bytes", "word_bytes",
                           "pad_bytes", "raw_bytes")}

    @property
    def ptr(self):
        if self._p is None:
            raise ValueError("blob already freed")
        return self._p

    def array(self) -> np.ndarray:
        """Zero-copy numpy view of the host blob bytes (valid until free)."""
        b = self.ptr.contents
        return np.ctypeslib.as_array(b.data, shape=(self.size,))

    def tobytes(self) -> bytes:
        return C.string_at(self.ptr.contents.data, self.size)

    def _descriptor(self, t: int) -> bytes:
        """Bytes of tensor t's descriptor, without a numpy view of the blob: the
        fused products read every job's shape and format several times a call,
        3.1-3.6 us a read by a view and 1 us by this."""
        data = self.ptr.contents.data
        t = operator.index(t)
        if not 0 <= t < self.n_tensors:
            raise IndexError(f"tensor {t} of a blob of {self.n_tensors}")
        return C.string_at(C.addressof(data.contents) + 64 + 96 * t, 96)

    def shape(self, t: int):
        """(rows, cols) of tensor t in symbol elements, from its descriptor in
        the blob header (blob format: 64-byte header, 96-byte descriptors with
        rows and cols at bytes 64 and 72); (0, 0) for an unshaped tensor."""
        return struct.unpack_from("<QQ", self._descriptor(t), 64)

    def dtype(self, t: int) -> str:
        """Storage format of tensor t (the descriptor's first u32)."""
        return _DTYPE_NAMES[struct.unpack_from("<I", self._descriptor(t))[0]]

    def payload_bytes(self) -> int:
        """Lane states + words + raw bytes (what the entropy bound is compared with)."""
        d = self.breakdown
        return d["state_bytes"] + d["word_bytes"] + d["raw_bytes"]

    def free(self):
        if self._p is not None:
            lib().wc_free(self._p)
            self._p = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def encode(tensors, chunk_bytes: int = 65536, lanes: int = 64, threads: int = 0, tile=(0, 0),
           codebook: str = "tensor", tile_order: int = 0) -> Blob:
    """wc_encode of a list of (dtype, host array[, (rows, cols)]) entries.

    The shape is in symbol elements (16-bit words, bytes or nibbles); `tile`
    = (tile_rows, tile_cols) cuts every tensor it divides into one chunk per
    tile (tile_order 0: row-major tiles, 1: column blocks, the wc_gemv layout).
    codebook "layer" shares one table among the tensors of a dtype.
    """
    keep = [_bytes(e[1]) for e in tensors]
    arr = (_Tensor * len(tensors))()
    for i, (e, b) in enumerate(zip(tensors, keep)):
        rows, cols = e[2] if len(e) > 2 and e[2] is not None else (0, 0)
        arr[i] = _Tensor(b.ctypes.data if b.size else None, b.size, DTYPES[e[0]], 0, rows, cols)
    prm = _Params(chunk_bytes, lanes, 12, threads, tile[0], tile[1], CODEBOOKS[codebook],
                  tile_order)
    out = C.POINTER(_Blob)()
    rc = lib().wc_encode(arr, len(tensors), C.byref(prm), C.byref(out))
    if rc:
        raise WcError("wc_encode", rc)
    return Blob(out)


def open_blob(data) -> Blob:
    """wc_open: validate and take a copy of blob bytes made elsewhere."""
    b = _bytes(np.frombuffer(data, np.uint8) if isinstance(data, (bytes, bytearray)) else data)
    out = C.POINTER(_Blob)()
    rc = lib().wc_open(b.ctypes.data, b.size, C.byref(out))
    if rc:
        raise WcError("wc_open", rc)
    return Blob(out)


def decode(blob: Blob, dev_blob: int, dev_dst, stream: int = 0, dev_err: int = 0) -> None:
    """wc_decode with raw device pointers (ints); asynchronous on `stream`."""
    ptrs = (C.c_void_p * max(1, len(dev_dst)))(*[p or None for p in dev_dst])
    rc = lib().wc_decode(blob.ptr, C.c_void_p(dev_blob), ptrs, len(dev_dst),
                         C.c_void_p(stream or None), C.c_void_p(dev_err or None))
    if rc:
        raise WcError("wc_decode", rc)


def gemv(blob: Blob, dev_blob: int, tensors, dev_x, m: int, dev_y, stream: int = 0,
         dev_err: int = 0) -> None:
    """wc_gemv with raw device pointers: y_i (m x N fp32) += x_i (m x K bf16) * W_i^T for
    each job i (tensors, dev_x, dev_y: equal-length lists), in one launch."""
    n = len(tensors)
    ts = (C.c_uint32 * max(n, 1))(*tensors)
    xs = (C.c_void_p * max(n, 1))(*[p or None for p in dev_x])
    ys = (C.c_void_p * max(n, 1))(*[p or None for p in dev_y])
    rc = lib().wc_gemv(blob.ptr, C.c_void_p(dev_blob), n, ts, xs, m, ys,
                       C.c_void_p(stream or None), C.c_void_p(dev_err or None))
    if rc:
        raise WcError("wc_gemv", rc)


def gemm_workspace_bytes(blob: Blob, tensors, dev_x, m: int) -> int:
    """wc_gemm_workspace_bytes: device bytes wc_gemm needs for these jobs (0 up
    to 64 rows of x; jobs with the same x share its packed copy)."""
    n = len(tensors)
    ts = (C.c_uint32 * max(n, 1))(*tensors)
    xs = (C.c_void_p * max(n, 1))(*[p or None for p in dev_x])
    out = C.c_uint64(0)
    rc = lib().wc_gemm_workspace_bytes(blob.ptr, n, ts, xs, m, C.byref(out))
    if rc:
        raise WcError("wc_gemm_workspace_bytes", rc)
    return out.value


def gemm(blob: Blob, dev_blob: int, tensors, dev_x, m: int, dev_y, workspace: int = 0,
         workspace_bytes: int = 0, stream: int = 0, dev_err: int = 0) -> None:
    """wc_gemm with raw device pointers: wc_gemv for up to 64 rows of x, the
    shared fused GEMM (packed x in the caller's workspace) above."""
    n = len(tensors)
    ts = (C.c_uint32 * max(n, 1))(*tensors)
    xs = (C.c_void_p * max(n, 1))(*[p or None for p in dev_x])
    ys = (C.c_void_p * max(n, 1))(*[p or None for p in dev_y])
    rc = lib().wc_gemm(blob.ptr, C.c_void_p(dev_blob), n, ts, xs, m, ys,
                       C.c_void_p(workspace or None), workspace_bytes,
                       C.c_void_p(stream or None), C.c_void_p(dev_err or None))
    if rc:
        raise WcError("wc_gemm", rc)


def gemm_i8(blob: Blob, dev_blob: int, tensors, dev_x, m: int, dev_y, stream: int = 0,
            dev_err: int = 0) -> None:
    """wc_gemm_i8 with raw device pointers: y_i (m x N int32) += x_i (m x K int8)
    * W_i^T (int8), exactly, in one launch."""
    n = len(tensors)
    ts = (C.c_uint32 * max(n, 1))(*tensors)
    xs = (C.c_void_p * max(n, 1))(*[p or None for p in dev_x])
    ys = (C.c_void_p * max(n, 1))(*[p or None for p in dev_y])
    rc = lib().wc_gemm_i8(blob.ptr, C.c_void_p(dev_blob), n, ts, xs, m, ys,
                          C.c_void_p(stream or None), C.c_void_p(dev_err or None))
    if rc:
        raise WcError("wc_gemm_i8", rc)


def gemv_mx(blob: Blob, dev_blob: int, tensors, dev_scales, dev_x, m: int, dev_y,
            stream: int = 0, dev_err: int = 0) -> None:
    """wc_gemv_mx with raw device pointers: y_i (m x N float) += x_i (m x K bf16)
    * W_i^T for MXFP4 W_i (e2m1 codes in the blob, e8m0 scales at dev_scales[i])."""
    n = len(tensors)
    ts = (C.c_uint32 * max(n, 1))(*tensors)
    ss = (C.c_void_p * max(n, 1))(*[p or None for p in dev_scales])
    xs = (C.c_void_p * max(n, 1))(*[p or None for p in dev_x])
    ys = (C.c_void_p * max(n, 1))(*[p or None for p in dev_y])
    rc = lib().wc_gemv_mx(blob.ptr, C.c_void_p(dev_blob), n, ts, ss, xs, m, ys,
                          C.c_void_p(stream or None), C.c_void_p(dev_err or None))
    if rc:
        raise WcError("wc_gemv_mx", rc)


def gemv_w4(blob: Blob, dev_blob: int, tensors, dev_scales, dev_zeros, dev_x, m: int, dev_y,
            stream: int = 0, dev_err: int = 0) -> None:
    """wc_gemv_w4 with raw device pointers: y_i += x_i * W_i^T for int4 W_i (packed
    codes as the blob's byte tensor, fp16 scales per 128 at dev_scales[i], zero
    points at dev_zeros[i] or 0 for two's-complement codes; dev_zeros None: all
    two's-complement)."""
    n = len(tensors)
    ts = (C.c_uint32 * max(n, 1))(*tensors)
    ss = (C.c_void_p * max(n, 1))(*[p or None for p in dev_scales])
    zs = None if dev_zeros is None else (C.c_void_p * max(n, 1))(*[p or None for p in dev_zeros])
    xs = (C.c_void_p * max(n, 1))(*[p or None for p in dev_x])
    ys = (C.c_void_p * max(n, 1))(*[p or None for p in dev_y])
    rc = lib().wc_gemv_w4(blob.ptr, C.c_void_p(dev_blob), n, ts, ss, zs, xs, m, ys,
                          C.c_void_p(stream or None), C.c_void_p(dev_err or None))
    if rc:
        raise WcError("wc_gemv_w4", rc)


def stream_bytes(dev_src: int, src_bytes: int, dev_dst: int, dst_bytes: int, blocks: int = 0,
                 stream: int = 0) -> int:
    """wc_stream (a measuring aid, no decoding): read src_bytes once and write
    dst_bytes once, non-temporal, on `stream`; returns the bytes it reads."""
    rd = C.c_uint64(0)
    rc = lib().wc_stream(C.c_void_p(dev_src or None), src_bytes, C.c_void_p(dev_dst or None),
                         dst_bytes, blocks, C.c_void_p(stream or None), C.byref(rd))
    if rc:
        raise WcError("wc_stream", rc)
    return rd.value


# --- torch plumbing: device memory and streams only ---------------------------

def to_device(blob: Blob, device="cuda"):
    """Copy the blob bytes into a new uint8 device tensor."""
    import torch
    host = torch.from_numpy(blob.array())
    return host.to(device)


def decode_torch(blob: Blob, dev_blob, outs=None, stream=None, err=None):
    """Decode into uint8 device tensors (allocated if `outs` is None).

    Returns the list of output tensors.  `err` (int32 device tensor of one
    element) receives the WC_DERR_* bits; the caller reads it after syncing.
    """
    import torch
    dev = dev_blob.device
    if outs is None:
        outs = [torch.empty(n, dtype=torch.uint8, device=dev) for n in blob.out_bytes]
    for o, n in zip(outs, blob.out_bytes):
        if o.numel() * o.element_size() < n or not o.is_contiguous():
            raise ValueError("output tensor too small or not contiguous")
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    decode(blob, dev_blob.data_ptr(), [o.data_ptr() if n else 0 for o, n in zip(outs, blob.out_bytes)],
           stream.cuda_stream, err.data_ptr() if err is not None else 0)
    return outs


def _zeros(blob: Blob, tensors, xs, m: int, dtype):
    """y of each job, m x N, cleared in one launch for all jobs: seven fills took
    10 us before the seven products of a 70B layer (395 us with them, 384 now)."""
    import torch
    ys = [torch.empty((m, blob.shape(t)[0]), dtype=dtype, device=x.device)
          for t, x in zip(tensors, xs)]
    if ys:
        torch._foreach_zero_(ys)
    return ys


def describe_errors(bits: int) -> list:
    return [name for b, name in DERR.items() if bits & b]


def gemv_torch(blob: Blob, dev_blob, tensors, xs, ys=None, stream=None, err=None):
    """Fused decode-GEMM into float32 tensors, one launch: ys[i] += xs[i] @ W_i^T for
    W_i = tensor tensors[i] (ys zeroed and returned if None)."""
    import torch
    m = xs[0].shape[0]
    for x in xs:
        if x.dtype != torch.bfloat16 or not x.is_contiguous() or x.shape[0] != m:
            raise ValueError("xs must be contiguous bfloat16 tensors with equal row counts")
    if ys is None:
        ys = _zeros(blob, tensors, xs, m, torch.float32)
    if stream is None:
        stream = torch.cuda.current_stream(xs[0].device)
    gemv(blob, dev_blob.data_ptr(), list(tensors), [x.data_ptr() for x in xs], m,
         [y.data_ptr() for y in ys], stream.cuda_stream, err.data_ptr() if err is not None else 0)
    return ys


# --- device-side analysis and encoder ----------------------------------------
# wc_dtensor has wc_tensor's layout, with a device pointer in the first field.

def _dtensors(entries):
    """ctypes wc_dtensor array of (dtype, device tensor[, (rows, cols)]) entries."""
    arr = (_Tensor * len(entries))()
    for i, e in enumerate(entries):
        x = e[1]
        if not x.is_contiguous():
            raise ValueError("device tensors must be contiguous")
        nbytes = x.numel() * x.element_size()
        rows, cols = e[2] if len(e) > 2 and e[2] is not None else (0, 0)
        arr[i] = _Tensor(x.data_ptr() if nbytes else None, nbytes, DTYPES[e[0]], 0, rows, cols)
    return arr


def _params(chunk_bytes, lanes, tile, codebook, tile_order):
    return _Params(chunk_bytes, lanes, 12, 0, tile[0], tile[1], CODEBOOKS[codebook], tile_order)


def analyze_device(dtype: str, x, workspace=None, stream=None) -> dict:
    """wc_analyze_device of a device tensor (synchronises `stream`)."""
    import torch
    t = _dtensors([(dtype, x)])
    if workspace is None:
        workspace = torch.empty(ANALYZE_WORKSPACE_BYTES, dtype=torch.uint8, device=x.device)
    if stream is None:
        stream = torch.cuda.current_stream(x.device)
    st = _Stats()
    rc = lib().wc_analyze_device(t, C.c_void_p(workspace.data_ptr()), workspace.numel(),
                                 C.c_void_p(stream.cuda_stream or None), C.byref(st))
    if rc:
        raise WcError("wc_analyze_device", rc)
    return _stats_dict(st)


def analyze_device_static(dtype: str, x, stream=None) -> dict:
    """wc_analyze_device_static of a tensor on the current device: no workspace,
    the bins are the library's own device array (synchronises `stream`)."""
    import torch
    t = _dtensors([(dtype, x)])
    if stream is None:
        stream = torch.cuda.current_stream(x.device)
    st = _Stats()
    rc = lib().wc_analyze_device_static(t, C.c_void_p(stream.cuda_stream or None), C.byref(st))
    if rc:
        raise WcError("wc_analyze_device_static", rc)
    return _stats_dict(st)


def encode_device_bounds(entries, chunk_bytes: int = 65536, lanes: int = 64, tile=(0, 0),
                         codebook: str = "tensor", tile_order: int = 0):
    """(blob capacity, workspace bytes) wc_encode_device needs.  `entries` are
    (dtype, nbytes[, (rows, cols)]) or (dtype, tensor[, shape]) entries."""
    arr = (_Tensor * len(entries))()
    for i, e in enumerate(entries):
        nb = e[1] if isinstance(e[1], int) else e[1].numel() * e[1].element_size()
        rows, cols = e[2] if len(e) > 2 and e[2] is not None else (0, 0)
        arr[i] = _Tensor(None, nb, DTYPES[e[0]], 0, rows, cols)
    prm = _params(chunk_bytes, lanes, tile, codebook, tile_order)
    cap, ws = C.c_uint64(), C.c_uint64()
    rc = lib().wc_encode_device_bounds(arr, len(entries), C.byref(prm), C.byref(cap), C.byref(ws))
    if rc:
        raise WcError("wc_encode_device_bounds", rc)
    return cap.value, ws.value


def encode_device(entries, chunk_bytes: int = 65536, lanes: int = 64, tile=(0, 0),
                  codebook: str = "tensor", tile_order: int = 0, blob=None, workspace=None,
                  size=None, stream=None):
    """wc_encode_device of (dtype, device tensor[, (rows, cols)]) entries.

    Returns (blob, size): a uint8 device tensor of the capacity the bounds
    give and an int64 device tensor of one element that receives the blob's
    size; both are valid after `stream` (default: the current one) syncs.
    """
    import torch
    dev = entries[0][1].device
    cap, wsb = encode_device_bounds([(e[0], e[1]) + tuple(e[2:]) for e in entries], chunk_bytes,
                                    lanes, tile, codebook, tile_order)
    if blob is None:
        blob = torch.empty(cap, dtype=torch.uint8, device=dev)
    if workspace is None:
        workspace = torch.empty(wsb, dtype=torch.uint8, device=dev)
    if size is None:
        size = torch.zeros(1, dtype=torch.int64, device=dev)
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    arr = _dtensors(entries)
    prm = _params(chunk_bytes, lanes, tile, codebook, tile_order)
    rc = lib().wc_encode_device(arr, len(entries), C.byref(prm), C.c_void_p(blob.data_ptr()),
                                blob.numel(), C.c_void_p(workspace.data_ptr()), workspace.numel(),
                                C.c_void_p(stream.cuda_stream or None),
                                C.c_void_p(size.data_ptr()))
    if rc:
        raise WcError("wc_encode_device", rc)
    return blob, size


def gemm_torch(blob: Blob, dev_blob, tensors, xs, ys=None, workspace=None, stream=None, err=None):
    """wc_gemm into float32 tensors: ys[i] += xs[i] @ W_i^T (ys zeroed and
    returned if None; the workspace is allocated if None)."""
    import torch
    m = xs[0].shape[0]
    for x in xs:
        if x.dtype != torch.bfloat16 or not x.is_contiguous() or x.shape[0] != m:
            raise ValueError("xs must be contiguous bfloat16 tensors with equal row counts")
    if ys is None:
        ys = _zeros(blob, tensors, xs, m, torch.float32)
    need = gemm_workspace_bytes(blob, list(tensors), [x.data_ptr() for x in xs], m)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=xs[0].device)
    if stream is None:
        stream = torch.cuda.current_stream(xs[0].device)
    gemm(blob, dev_blob.data_ptr(), list(tensors), [x.data_ptr() for x in xs], m,
         [y.data_ptr() for y in ys], workspace.data_ptr(), workspace.numel(), stream.cuda_stream,
         err.data_ptr() if err is not None else 0)
    return ys


def gemm_i8_torch(blob: Blob, dev_blob, tensors, xs, ys=None, stream=None, err=None):
    """wc_gemm_i8 into int32 tensors: ys[i] += xs[i] @ W_i^T for int8 xs and
    int8 W_i = tensor tensors[i] (ys zeroed and returned if None)."""
    import torch
    m = xs[0].shape[0]
    for x in xs:
        if x.dtype != torch.int8 or not x.is_contiguous() or x.shape[0] != m:
            raise ValueError("xs must be contiguous int8 tensors with equal row counts")
    if ys is None:
        ys = _zeros(blob, tensors, xs, m, torch.int32)
    if stream is None:
        stream = torch.cuda.current_stream(xs[0].device)
    gemm_i8(blob, dev_blob.data_ptr(), list(tensors), [x.data_ptr() for x in xs], m,
            [y.data_ptr() for y in ys], stream.cuda_stream, err.data_ptr() if err is not None else 0)
    return ys


def _codes_shape(blob: Blob, t: int):
    """(N, K) of a 4-bit weight tensor in codes: a nibble tensor's own shape, or
    twice the columns of a byte tensor holding the packed codes."""
    n, k = blob.shape(t)
    if blob.dtype(t) == "u8":
        k *= 2
    return n, k


def _check_jobs(blob: Blob, tensors, xs, m: int):
    """xs: one contiguous bf16 m x K tensor per job, K the weights' code count."""
    import torch
    if len(xs) != len(tensors):
        raise ValueError("one x per job")
    for t, x in zip(tensors, xs):
        if x.dtype != torch.bfloat16 or not x.is_contiguous() or x.dim() != 2 or x.shape[0] != m:
            raise ValueError("xs must be contiguous 2-D bfloat16 tensors with equal row counts")
        if not 0 <= t < blob.n_tensors:
            raise ValueError(f"tensor index {t} out of range")
        k = _codes_shape(blob, t)[1]
        if x.shape[1] != k:
            raise ValueError(f"tensor {t}: x has {x.shape[1]} columns, the weights {k}")


def gemv_mx_torch(blob: Blob, dev_blob, tensors, scales, xs, ys=None, stream=None, err=None):
    """wc_gemv_mx into float32 tensors: ys[i] += xs[i] @ W_i^T for MXFP4 W_i =
    tensor tensors[i] with e8m0 scales `scales[i]` (uint8 device tensors of
    N x K/32); ys zeroed and returned if None."""
    import torch
    m = xs[0].shape[0]
    _check_jobs(blob, tensors, xs, m)
    if len(scales) != len(tensors):
        raise ValueError("one scale tensor per job")
    for t, sc in zip(tensors, scales):
        n, k = _codes_shape(blob, t)
        if sc.dtype != torch.uint8 or not sc.is_contiguous():
            raise ValueError("scales must be contiguous uint8 tensors")
        if sc.numel() != n * (k // 32):
            raise ValueError(f"tensor {t}: {sc.numel()} scale bytes, the weights need N * K/32 = "
                             f"{n * (k // 32)}")
    if ys is None:
        ys = _zeros(blob, tensors, xs, m, torch.float32)
    if stream is None:
        stream = torch.cuda.current_stream(xs[0].device)
    gemv_mx(blob, dev_blob.data_ptr(), list(tensors), [sc.data_ptr() for sc in scales],
            [x.data_ptr() for x in xs], m, [y.data_ptr() for y in ys], stream.cuda_stream,
            err.data_ptr() if err is not None else 0)
    return ys


def gemv_w4_torch(blob: Blob, dev_blob, tensors, scales, zeros, xs, ys=None, stream=None,
                  err=None):
    """wc_gemv_w4 into float32 tensors: ys[i] += xs[i] @ W_i^T for int4 W_i with fp16
    scales `scales[i]` (device tensors holding N x K/128 binary16 words, of any
    element type) and zero points `zeros[i]` (uint8 device tensors of one byte per
    group, or None for two's-complement codes; `zeros` None: all two's-complement);
    ys zeroed and returned if None.  Every tensor's size is checked against the
    weights' shape before the launch (ValueError), since the kernel sizes its reads
    from the blob, not from the tensors passed."""
    import torch
    m = xs[0].shape[0]
    _check_jobs(blob, tensors, xs, m)
    if len(scales) != len(tensors) or (zeros is not None and len(zeros) != len(tensors)):
        raise ValueError("one scale tensor (and one zero-point entry, if any) per job")
    for i, t in enumerate(tensors):
        n, k = _codes_shape(blob, t)
        sc = scales[i]
        if not sc.is_contiguous() or sc.data_ptr() % 2:
            raise ValueError("scales must be contiguous and 2-byte aligned")
        if sc.numel() * sc.element_size() != 2 * n * (k // 128):
            raise ValueError(f"tensor {t}: {sc.numel() * sc.element_size()} bytes of scales, the "
                             f"weights need N * K/128 = {n * (k // 128)} fp16 words")
        z = None if zeros is None else zeros[i]
        if z is not None:
            if z.dtype != torch.uint8 or not z.is_contiguous():
                raise ValueError("zero points must be contiguous uint8 tensors, one byte a group")
            if z.numel() != n * (k // 128):
                raise ValueError(f"tensor {t}: {z.numel()} zero points, the weights need one "
                                 f"byte per group, N * K/128 = {n * (k // 128)} (packed "
                                 "nibbles must be unpacked first)")
    if ys is None:
        ys = _zeros(blob, tensors, xs, m, torch.float32)
    if stream is None:
        stream = torch.cuda.current_stream(xs[0].device)
    zp = None if zeros is None else [z.data_ptr() if z is not None else 0 for z in zeros]
    gemv_w4(blob, dev_blob.data_ptr(), list(tensors), [s.data_ptr() for s in scales], zp,
            [x.data_ptr() for x in xs], m, [y.data_ptr() for y in ys], stream.cuda_stream,
            err.data_ptr() if err is not None else 0)
    return ys


# --- 8-bit integer layers -----------------------------------------------------
# The layers of a decoded int8 checkpoint.  Matrices are int8 (or the uint8 buffers
# decode_torch fills: the same bytes), activations, scales and results bfloat16,
# float16 or float32.

_NO_CONTEXT = contextlib.nullcontext()
SCORES = {"softmax": 0, "sigmoid": 1}
_floats, _ints = {}, ()
_FP32 = 8  # WC_FP32
_EINVAL = -1  # WC_EINVAL: here for sizes that ctypes would cut to 32 bits


def _types():
    """C types of the float element types; filled at the first call, with torch."""
    global _floats, _ints
    if not _floats:
        import torch
        _ints = (torch.int8, torch.uint8)
        _floats = {torch.bfloat16: 1, torch.float16: 2, torch.float32: _FP32}
    return _floats


def _float_type(t, what: str) -> int:
    code = _types().get(t.dtype)
    if code is None:
        raise ValueError(f"{what} must be bfloat16, float16 or float32")
    return code


# The first tensor of a call says on which device it runs (get_device: -1 for host memory);
# every other one has to be there.

def _rows(t, what: str, dev: int, cols: int = -1) -> int:
    """Row stride, in elements, of a 2-D tensor on device `dev` whose rows are contiguous."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or dev < 0 or t.get_device() != dev:
        raise ValueError(f"{what} must be a 2-D tensor on {'a device' if dev < 0 else f'device {dev}'}")
    if cols >= 0 and shape[1] != cols:
        raise ValueError(f"{what} has {shape[1]} columns, not {cols}")
    if stride[1] != 1 and shape[1] > 1:
        raise ValueError(f"{what}: the elements of a row must be next to each other")
    return stride[0] if shape[0] > 1 else shape[1]


def _vector(t, n: int, what: str, dev: int) -> int:
    if t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{what} must be {n} contiguous elements on device {dev}")
    return _float_type(t, what)


def _codes(t, what: str):
    _types()
    if t.dtype not in _ints:
        raise ValueError(f"{what} must be int8 codes")
    return t


def _stream_of(stream, device):
    """The stream handle to launch on, and the context in which to launch, so that the
    device is the current one, and to allocate what the launch uses, so that the allocator
    knows the stream that uses it."""
    import torch
    if stream is None:
        index = device.index
        return torch._C._cuda_getCurrentRawStream(index), \
            _NO_CONTEXT if torch._C._cuda_getDevice() == index else torch.cuda.device(index)
    if stream.device_index != device.index:
        raise ValueError(f"the stream must be one of device {device.index}")
    return stream.cuda_stream, torch.cuda.stream(stream)


def _workspace(workspace, need: int, device):
    import torch
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device) if need else None
    if workspace.numel() * workspace.element_size() < need or not workspace.is_contiguous() or \
            workspace.get_device() != device.index:
        raise ValueError(f"the workspace needs {need} contiguous bytes on device {device.index}")
    return workspace


def _ptr(t):
    return None if t is None else t.data_ptr()


def _size(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def i8_row_bytes(k: int) -> int:
    """WC_I8_ROW_BYTES: bytes of a row of quantised activations."""
    return (k + 127) // 128 * 128


def quantize_i8_torch(x, q=None, scale=None, stream=None):
    """wc_quantize_i8 of a 2-D tensor: (q, scale), q int8 of m x i8_row_bytes(k) (zero
    past column k) and scale float32 of m; the row's values are q * scale."""
    import torch
    dev = x.get_device()
    ld = _rows(x, "x", dev)
    dt = _float_type(x, "x")
    m, k = x.shape
    if (m | k) >> 32:
        raise WcError("wc_quantize_i8", _EINVAL)
    st, where = _stream_of(stream, x.device)
    with where:
        if q is None:
            q = torch.empty((m, i8_row_bytes(k)), dtype=torch.int8, device=x.device)
        if scale is None:
            scale = torch.empty(m, dtype=torch.float32, device=x.device)
        if tuple(q.shape) != (m, i8_row_bytes(k)) or q.dtype != torch.int8 or \
                not q.is_contiguous() or q.get_device() != dev:
            raise ValueError(f"q must be a contiguous int8 tensor of {m} x {i8_row_bytes(k)} on device {dev}")
        if _vector(scale, m, "scale", dev) != _FP32:
            raise ValueError("scale must be float32")
        rc = lib().wc_quantize_i8(x.data_ptr(), dt, m, k, ld, q.data_ptr(), scale.data_ptr(), st)
    if rc:
        raise WcError("wc_quantize_i8", rc)
    return q, scale


_JOB = struct.Struct("=6QI3i")  # wc_i8_job


def _i8_jobs(m: int, k: int, ws, scales, biases, ys, dtype, dev: int):
    """The wc_i8_job array, packed, and the ys (allocated where None)."""
    n_jobs = len(ws)
    if len(scales) != n_jobs or (biases is not None and len(biases) != n_jobs) or \
            (ys is not None and len(ys) != n_jobs):
        raise ValueError("one scale tensor, bias entry and y a matrix")
    floats = _types()
    jobs, out = [], []
    yt = floats.get(dtype)
    for i in range(n_jobs):
        w, s = ws[i], scales[i]
        # (each look at a tensor costs the host as much as a microsecond's tenth)
        shape, stride = w.shape, w.stride()
        if len(shape) != 2 or shape[1] != k or w.get_device() != dev or (stride[1] != 1 and k > 1):
            _rows(w, "w", dev, k)
        if w.dtype not in _ints:
            raise ValueError("w must be int8 codes")
        n = shape[0]
        ldw = stride[0] if n > 1 else k
        st = _vector(s, n, "a matrix's scale", dev)
        b = None if biases is None else biases[i]
        bp, bt = (0, 0) if b is None else (b.data_ptr(), _vector(b, n, "a bias", dev))
        if ys is None:
            y, ldy = w.new_empty((m, n), dtype=dtype), n
        else:
            y = ys[i]
            if y.shape != (m, n):
                raise ValueError(f"y must be {m} x {n}")
            ldy = _rows(y, "y", dev)
            yt = floats.get(y.dtype)
        if yt is None:
            raise ValueError("y must be bfloat16, float16 or float32")
        out.append(y)
        if n >> 32:
            raise WcError("wc_matmul_i8", _EINVAL)
        jobs.append(_JOB.pack(w.data_ptr(), s.data_ptr(), bp, y.data_ptr(), ldw, ldy, n, st, bt, yt))
    return b"".join(jobs), out


def matmul_i8_torch(q, scale, k: int, ws, scales, biases=None, ys=None, dtype=None,
                    workspace=None, stream=None):
    """wc_matmul_i8: (q * scale) @ (W_i * scales_i)^T + biases_i for each int8 W_i (n_i x
    k) of `ws`, with q and scale from quantize_i8_torch.  ys (of any float type, rows
    contiguous) are allocated in `dtype` (bfloat16 if None) where None."""
    import torch
    dev, m = q.get_device(), q.shape[0]
    if dev < 0 or q.dtype != torch.int8 or not q.is_contiguous() or \
            tuple(q.shape) != (m, i8_row_bytes(k)):
        raise ValueError(f"q must be a contiguous int8 device tensor of {i8_row_bytes(k)} columns")
    if _vector(scale, m, "scale", dev) != _FP32:
        raise ValueError("scale must be float32")
    if (m | k) >> 32:
        raise WcError("wc_matmul_i8", _EINVAL)
    st, where = _stream_of(stream, q.device)
    need = C.c_uint64(0)
    with where:
        jobs, ys = _i8_jobs(m, k, ws, scales, biases, ys, dtype or torch.bfloat16, dev)
        rc = lib().wc_matmul_i8_workspace_bytes(m, k, len(ws), jobs, C.byref(need))
        if not rc:
            workspace = _workspace(workspace, need.value, q.device)
            rc = lib().wc_matmul_i8(q.data_ptr(), scale.data_ptr(), m, k, len(ws), jobs,
                                    _ptr(workspace), _size(workspace), st)
    if rc:
        raise WcError("wc_matmul_i8", rc)
    return ys


def linear_i8_torch(x, ws, scales, biases=None, ys=None, dtype=None, workspace=None,
                    stream=None):
    """wc_linear_i8: x quantised per row, then as matmul_i8_torch; `dtype` defaults to
    x's type."""
    dev = x.get_device()
    ld = _rows(x, "x", dev)
    dt = _float_type(x, "x")
    m, k = x.shape
    if (m | k) >> 32:
        raise WcError("wc_linear_i8", _EINVAL)
    st, where = _stream_of(stream, x.device)
    need = C.c_uint64(0)
    with where:
        jobs, ys = _i8_jobs(m, k, ws, scales, biases, ys, dtype or x.dtype, dev)
        # one or two rows mostly need no workspace, and the call refuses those that do
        if m <= 2 and workspace is None and \
                not lib().wc_linear_i8(x.data_ptr(), dt, m, k, ld, len(ws), jobs, None, 0, st):
            return ys
        rc = lib().wc_linear_i8_workspace_bytes(m, k, len(ws), jobs, C.byref(need))
        if not rc:
            workspace = _workspace(workspace, need.value, x.device)
            rc = lib().wc_linear_i8(x.data_ptr(), dt, m, k, ld, len(ws), jobs, _ptr(workspace),
                                    _size(workspace), st)
    if rc:
        raise WcError("wc_linear_i8", rc)
    return ys


# What wc_route writes: ids and weights (tokens x k), offsets (experts + 1), order
# (tokens * k slots sorted by expert).
Routing = namedtuple("Routing", "ids weights offsets order")


def route_torch(logits, k: int, score: str = "softmax", bias=None, groups: int = 1,
                top_groups: int = 1, group_top: int = 1, renormalize: bool = True,
                scale: float = 1.0, out=None, workspace=None, stream=None) -> Routing:
    """wc_route of a router's logits (tokens x experts); `bias` float32 of experts;
    `out` a Routing to write into."""
    import torch
    on = logits.get_device()
    ld = _rows(logits, "logits", on)
    dt = _float_type(logits, "logits")
    tokens, experts = logits.shape
    if score not in SCORES:
        raise ValueError(f"score must be one of {sorted(SCORES)}")
    if bias is not None and _vector(bias, experts, "bias", on) != _FP32:
        raise ValueError("bias must be float32")
    if (tokens | experts | k | groups | top_groups | group_top) >> 32:
        raise WcError("wc_route", _EINVAL)
    dev = logits.device
    st, where = _stream_of(stream, dev)
    params = _RouteParams(experts, k, SCORES[score], int(renormalize), groups, top_groups,
                          group_top, scale)
    need = C.c_uint64(0)
    # few slots need no workspace
    rc = 0 if 0 < tokens * k <= 2048 and workspace is None else \
        lib().wc_route_workspace_bytes(tokens, C.byref(params), C.byref(need))
    if rc:
        raise WcError("wc_route", rc)
    with where:
        if out is None:
            new = logits.new_empty
            out = Routing(new((tokens, k), dtype=torch.int32), new((tokens, k), dtype=torch.float32),
                          new(experts + 1, dtype=torch.int32), new(tokens * k, dtype=torch.int32))
        else:
            _check_routing(out, tokens, k, experts, on)
        workspace = _workspace(workspace, need.value, dev)
        rc = lib().wc_route(logits.data_ptr(), dt, tokens, ld, C.byref(params), _ptr(bias),
                            *(t.data_ptr() for t in out), _ptr(workspace), _size(workspace), st)
    if rc:
        raise WcError("wc_route", rc)
    return out


def _check_routing(r, tokens: int, k: int, experts: int, dev: int):
    import torch
    for t, shape, dtype, name in ((r.ids, (tokens, k), torch.int32, "ids"),
                                  (r.weights, (tokens, k), torch.float32, "weights"),
                                  (r.offsets, (experts + 1,), torch.int32, "offsets"),
                                  (r.order, (tokens * k,), torch.int32, "order")):
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != dev:
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of {shape} on device {dev}")


def _bank(w, scale, experts: int, n: int, k: int, what: str, dev: int):
    _codes(w, what)
    stride = w.stride()
    if w.shape != (experts, n, k) or w.get_device() != dev or (k > 1 and stride[2] != 1) or \
            (n > 1 and stride[1] != k):
        raise ValueError(f"{what} must be {experts} x {n} x {k} codes on device {dev}, contiguous in each "
                         "expert")
    if scale.shape != (experts, n):
        raise ValueError(f"the scales of {what} must be {experts} x {n}")
    return _I8Experts(w.data_ptr(), scale.data_ptr(), stride[0] if experts > 1 else n * k,
                      _vector(scale, experts * n, f"the scales of {what}", dev), 0)


def experts_i8_torch(x, routing: Routing, gate, gate_scale, up, up_scale, down, down_scale,
                     y=None, workspace=None, stream=None):
    """wc_experts_i8: the feed-forward of a mixture layer.  x tokens x hidden; gate, up
    int8 of experts x ffn x hidden, down of experts x hidden x ffn, with scales of
    experts x rows; y of x's type."""
    import torch
    dev = x.get_device()
    ld = _rows(x, "x", dev)
    dt = _float_type(x, "x")
    tokens, hidden = x.shape
    if gate.dim() != 3 or routing.ids.dim() != 2:
        raise ValueError("gate must be experts x ffn x hidden, the ids tokens x k")
    experts, ffn = gate.shape[:2]
    k = routing.ids.shape[1]
    if (tokens | k | experts | hidden | ffn) >> 32:
        raise WcError("wc_experts_i8", _EINVAL)
    _check_routing(routing, tokens, k, experts, dev)
    banks = (_bank(gate, gate_scale, experts, ffn, hidden, "gate", dev),
             _bank(up, up_scale, experts, ffn, hidden, "up", dev),
             _bank(down, down_scale, experts, hidden, ffn, "down", dev))
    st, where = _stream_of(stream, x.device)
    need = C.c_uint64(0)
    rc = lib().wc_experts_i8_workspace_bytes(tokens, k, experts, hidden, ffn, C.byref(need))
    if rc:
        raise WcError("wc_experts_i8", rc)
    with where:
        if y is None:
            y = x.new_empty((tokens, hidden))
        workspace = _workspace(workspace, need.value, x.device)
        if tuple(y.shape) != (tokens, hidden) or y.dtype != x.dtype:
            raise ValueError(f"y must be {tokens} x {hidden} of x's type")
        ldy = _rows(y, "y", dev)
        rc = lib().wc_experts_i8(x.data_ptr(), dt, tokens, ld, k, experts, hidden, ffn,
                                 *(t.data_ptr() for t in routing), *(C.byref(b) for b in banks),
                                 y.data_ptr(), ldy, _ptr(workspace), _size(workspace), st)
    if rc:
        raise WcError("wc_experts_i8", rc)
    return y
