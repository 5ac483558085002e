"""ctypes binding of libesparse.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels; torch is used for device memory and
for the current stream.  There is no fallback: if the shared library is missing, loading fails.
Names follow include/esparse.h.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

F16, BF16, F32 = 0, 1, 2
MX_FP4, MX_FP8 = 0, 1   # microscaled formats
_ACT_16 = 2             # activations of mx_gemm in 16 bits
MAX_TOP = 32            # alternatives of token_logprobs
USE_ENTROPY, USE_NORM, USE_GNS, USE_LBS, USE_ALL = 1, 2, 4, 8, 15

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libesparse.so")
_lib = None


class EsparseError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"esparse error {code}: {message}")
        self.code = code


class _Opts(C.Structure):
    _fields_ = [("n_keep", C.c_int), ("m_group", C.c_int), ("block", C.c_int), ("bins", C.c_int),
                ("alpha", C.c_double), ("flags", C.c_uint), ("max_swaps", C.c_longlong)]


def load_library():
    """Load libesparse.so (built by __graft_entry__.build()).  Raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python __graft_entry__.py` (there is no fallback path)")
    lib = C.CDLL(_LIB_PATH)
    vp, ll, i32, sz = C.c_void_p, C.c_longlong, C.c_int, C.c_size_t
    P = C.POINTER
    sig = {
        "esparse_create": (i32, [P(vp), i32, vp]),
        "esparse_destroy": (None, [vp]),
        "esparse_set_stream": (i32, [vp, vp]),
        "esparse_last_error": (C.c_char_p, [vp]),
        "esparse_version": (C.c_char_p, []),
        "esparse_channel_stats": (i32, [vp, vp, ll, ll, i32, i32, vp, vp]),
        "esparse_prune": (i32, [vp, vp, ll, vp, ll, ll, i32, P(_Opts), vp, vp, vp, vp, vp]),
        "esparse_prune_with_scores": (i32, [vp, vp, vp, ll, ll, i32, P(_Opts), vp, vp, vp, vp]),
        "esparse_output_error": (i32, [vp, vp, vp, ll, ll, i32, vp, vp]),
        "esparse_matrix_rate": (i32, [vp, i32, i32, i32, i32, P(C.c_double)]),
        "esparse_read_rate": (i32, [vp, sz, P(C.c_double)]),
        "esparse_spmm_group_workspace": (i32, [i32, ll, ll, ll, P(sz)]),
        "esparse_spmm_group": (i32, [vp, i32, P(vp), ll, P(vp), P(vp), ll, ll, i32, i32, i32, P(vp), vp, sz, i32]),
        "esparse_dense_gemm_group": (i32, [vp, i32, P(vp), ll, P(vp), ll, ll, i32, P(vp), vp, sz, i32]),
        "esparse_stage_activations_group": (i32, [vp, i32, P(vp), ll, P(vp), ll, ll, i32, i32, i32, vp, sz, i32]),
        "esparse_spmm_group_staged": (i32, [vp, i32, ll, P(vp), ll, ll, i32, i32, i32, P(vp), vp, sz, i32]),
        "esparse_compressed_size": (i32, [ll, ll, i32, i32, i32, P(sz), P(sz), P(sz)]),
        "esparse_compress": (i32, [vp, vp, vp, vp, ll, ll, i32, i32, i32, vp, vp, vp]),
        "esparse_spmm_workspace": (i32, [ll, ll, ll, i32, P(sz)]),
        "esparse_spmm": (i32, [vp, vp, ll, vp, vp, ll, ll, i32, i32, i32, vp, vp, sz, i32]),
        "esparse_spmm_static": (i32, [vp, vp, ll, vp, vp, ll, ll, i32, i32, i32, vp, i32]),
        "esparse_stage_activations": (i32, [vp, vp, ll, vp, ll, ll, i32, vp, sz]),
        "esparse_spmm_staged": (i32, [vp, ll, vp, ll, ll, i32, i32, i32, vp, vp, sz, i32]),
        "esparse_dense_gemm_staged": (i32, [vp, ll, vp, ll, ll, i32, vp, vp, sz, i32]),
        "esparse_spmm_num_variants": (i32, []),
        "esparse_spmm_variant_name": (C.c_char_p, [i32]),
        "esparse_dense_packed_size": (i32, [ll, ll, P(sz)]),
        "esparse_dense_pack": (i32, [vp, vp, ll, ll, i32, vp]),
        "esparse_dense_gemm": (i32, [vp, vp, ll, vp, ll, ll, i32, vp, vp, sz, i32]),
        "esparse_tune": (i32, [vp, ll, ll, ll, i32, i32, P(i32), P(C.c_float)]),
        "esparse_tune_group": (i32, [vp, i32, ll, ll, ll, i32, i32, P(i32), P(C.c_float)]),
        "esparse_tune_save": (i32, [vp, C.c_char_p]),
        "esparse_tune_load": (i32, [vp, C.c_char_p]),
        "esparse_mx_size": (i32, [ll, ll, i32, P(sz), P(sz)]),
        "esparse_mx_quantize": (i32, [vp, vp, ll, ll, ll, i32, i32, vp, vp]),
        "esparse_mx_dequantize": (i32, [vp, vp, vp, ll, ll, i32, i32, vp]),
        "esparse_mx_packed_size": (i32, [ll, ll, P(sz)]),
        "esparse_mx_pack": (i32, [vp, vp, vp, ll, ll, vp]),
        "esparse_mx_gemm_workspace": (i32, [ll, ll, ll, i32, i32, P(sz)]),
        "esparse_mx_gemm": (i32, [vp, vp, vp, ll, ll, i32, i32, vp, ll, ll, i32, vp, vp, sz]),
        "esparse_rms_norm": (i32, [vp, vp, ll, vp, ll, vp, ll, ll, C.c_double, i32, vp, vp, i32, vp, vp]),
        "esparse_token_logprobs_workspace": (i32, [ll, ll, i32, i32, P(sz)]),
        "esparse_token_logprobs": (i32, [vp, vp, ll, ll, ll, i32, vp, i32, vp, vp, vp, vp, vp, sz]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


EXPORTED = ["esparse_create", "esparse_destroy", "esparse_set_stream", "esparse_last_error",
            "esparse_version", "esparse_channel_stats", "esparse_prune", "esparse_prune_with_scores", "esparse_output_error",
            "esparse_matrix_rate", "esparse_read_rate",
            "esparse_spmm_group_workspace", "esparse_spmm_group", "esparse_dense_gemm_group",
            "esparse_stage_activations_group", "esparse_spmm_group_staged",
            "esparse_compressed_size", "esparse_compress", "esparse_spmm_workspace", "esparse_spmm", "esparse_spmm_static",
            "esparse_stage_activations", "esparse_spmm_staged", "esparse_dense_gemm_staged",
            "esparse_spmm_num_variants", "esparse_spmm_variant_name", "esparse_dense_packed_size",
            "esparse_dense_pack", "esparse_dense_gemm", "esparse_tune", "esparse_tune_group", "esparse_tune_save",
            "esparse_tune_load", "esparse_mx_size", "esparse_mx_quantize", "esparse_mx_dequantize", "esparse_mx_packed_size",
            "esparse_mx_pack", "esparse_mx_gemm_workspace", "esparse_mx_gemm", "esparse_rms_norm",
            "esparse_token_logprobs_workspace", "esparse_token_logprobs"]


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return F16
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


_CODES = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}


_EMPTY = torch.empty_strided


def _code(dtype: torch.dtype, name: str, f32: bool = False) -> int:
    """The library's number of a type that a call takes."""
    code = _CODES.get(dtype)
    if code is None or (code == F32 and not f32):
        raise TypeError(f"{name}: unsupported dtype {dtype}")
    return code


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_PTRS = [None] + [C.c_void_p * n for n in range(1, 5)]  # arrays of a group call's pointers


def _ptrs(ts):
    n = len(ts)
    return (_PTRS[n] if 0 < n < 5 else C.c_void_p * n)(*[_ptr(t) for t in ts])


def compressed_size(N: int, K: int, n: int, m: int, dtype: int = F16):
    lib = load_library()
    a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
    rc = lib.esparse_compressed_size(N, K, n, m, dtype, C.byref(a), C.byref(b), C.byref(c))
    if rc:
        raise EsparseError(rc, "esparse_compressed_size")
    return a.value, b.value, c.value


def spmm_workspace(M: int, N: int, K: int, variant: int = -1) -> int:
    lib = load_library()
    a = C.c_size_t()
    rc = lib.esparse_spmm_workspace(M, N, K, variant, C.byref(a))
    if rc:
        raise EsparseError(rc, "esparse_spmm_workspace")
    return a.value


def _group_workspace(count: int, M: int, N: int, K: int) -> int:
    a = C.c_size_t(0)
    rc = load_library().esparse_spmm_group_workspace(count, M, N, K, C.byref(a))
    if rc:
        raise EsparseError(rc, "esparse_spmm_group_workspace: bad arguments")
    return a.value


def mx_size(R: int, K: int, fmt: int):
    """(bytes of the codes, bytes of the scales) of R rows of K channels."""
    a, b = C.c_size_t(), C.c_size_t()
    rc = load_library().esparse_mx_size(R, K, fmt, C.byref(a), C.byref(b))
    if rc:
        raise EsparseError(rc, f"esparse_mx_size: R = {R}, K = {K}, format {fmt}")
    return a.value, b.value


def mx_packed_size(N: int, K: int) -> int:
    a = C.c_size_t()
    rc = load_library().esparse_mx_packed_size(N, K, C.byref(a))
    if rc:
        raise EsparseError(rc, f"esparse_mx_packed_size: N = {N}, K = {K}")
    return a.value


def mx_gemm_workspace(M: int, N: int, K: int, act: int, aligned: bool = True) -> int:
    a = C.c_size_t()
    rc = load_library().esparse_mx_gemm_workspace(M, N, K, act, int(aligned), C.byref(a))
    if rc:
        raise EsparseError(rc, f"esparse_mx_gemm_workspace: M = {M}, N = {N}, K = {K}, activations {act}")
    return a.value


def token_logprobs_workspace(R: int, V: int, dtype: int, top: int) -> int:
    a = C.c_size_t()
    rc = load_library().esparse_token_logprobs_workspace(R, V, dtype, top, C.byref(a))
    if rc:
        raise EsparseError(rc, f"esparse_token_logprobs_workspace: R = {R}, V = {V}, dtype {dtype}, top = {top}")
    return a.value


# for the calls: sizes asked for before, a function of their arguments alone (typed: 16.0 is not the 16 that was asked for)
_known_size = functools.lru_cache(4096, typed=True)(compressed_size)
_known_workspace = functools.lru_cache(4096, typed=True)(spmm_workspace)
_known_group_workspace = functools.lru_cache(4096, typed=True)(_group_workspace)
_known_mx_packed_size = functools.lru_cache(4096, typed=True)(mx_packed_size)
_known_mx_gemm_workspace = functools.lru_cache(4096, typed=True)(mx_gemm_workspace)
_known_logprobs_workspace = functools.lru_cache(4096, typed=True)(token_logprobs_workspace)


def dense_packed_size(N: int, K: int) -> int:
    lib = load_library()
    a = C.c_size_t()
    rc = lib.esparse_dense_packed_size(N, K, C.byref(a))
    if rc:
        raise EsparseError(rc, "esparse_dense_packed_size")
    return a.value


def num_variants() -> int:
    return load_library().esparse_spmm_num_variants()


def variant_name(v: int) -> str:
    return load_library().esparse_spmm_variant_name(v).decode()


@dataclass
class PruneOpts:
    n_keep: int = 2
    m_group: int = 4
    block: int = 64
    bins: int = 100
    alpha: float = 1.0
    flags: int = USE_ALL
    max_swaps: int = 0

    def _c(self) -> _Opts:
        return _Opts(self.n_keep, self.m_group, self.block, self.bins, float(self.alpha), self.flags,
                     self.max_swaps)


@dataclass
class PruneResult:
    perm: torch.Tensor          # int32 [K] device
    mask: torch.Tensor          # uint8 [N, K] device, re-ordered channel order
    score: Optional[np.ndarray]  # float64 [K] host
    swaps: Optional[np.ndarray]  # int64 [K / block] host
    retained: Optional[float]


@dataclass
class Compressed:
    values: Optional[torch.Tensor]
    meta: Optional[torch.Tensor]
    native: Optional[torch.Tensor]  # uint8 [native_bytes]
    N: int
    K: int
    n_keep: int
    m_group: int
    dtype: int


@dataclass
class MX:
    """Rows of microscaled numbers (include/esparse.h)."""
    data: torch.Tensor    # uint8 [R, Kp / 2] or [R, Kp], Kp = K rounded up to 128
    scales: torch.Tensor  # uint8 [Kp / 128, R, 4]
    K: int
    fmt: int              # MX_FP4 or MX_FP8


@dataclass
class MXWeight:
    """Weights in microscaled 4 bits, in the order mx_gemm streams them."""
    packed: torch.Tensor  # uint8 [mx_packed_size(N, K)]
    N: int
    K: int


@dataclass
class TokenLogprobs:
    logprob: Optional[torch.Tensor]       # float32 [R]
    entropy: torch.Tensor                 # float32 [R]
    top_ids: Optional[torch.Tensor]       # int32 [R, top]
    top_logprobs: Optional[torch.Tensor]  # float32 [R, top]


def _raw_stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)  # without the Stream object


class Context:
    """One library context bound to a device and (per call) to torch's current stream."""

    def __init__(self, device: int = 0):
        self._lib = load_library()
        self._h = C.c_void_p()
        rc = self._lib.esparse_create(C.byref(self._h), device, None)
        if rc:
            raise EsparseError(rc, "esparse_create")
        self.device = device
        self._on = torch.device("cuda", device)
        self._ws = None
        self._ws_at, self._ws_room = 0, -1  # the workspace's first aligned address and the bytes from there (-1: no workspace yet)
        self._stream = None              # the stream the library knows

    def close(self):
        if self._h:
            self._lib.esparse_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers ------------------------------------------------------------------------------
    def _check(self, rc: int):
        if rc:
            raise EsparseError(rc, self._lib.esparse_last_error(self._h).decode())

    def _sync_stream(self):
        if torch.cuda.is_initialized():
            s = _raw_stream(self.device)
        elif torch.cuda.is_available():
            s = torch.cuda.current_stream(self.device).cuda_stream
        else:
            return
        if s != self._stream:
            self._lib.esparse_set_stream(self._h, s)
            self._stream = s

    def _scratch(self, nbytes: int) -> int:
        """Address of the context's workspace, of at least nbytes, 256-byte aligned."""
        if self._ws_room < nbytes:
            self._ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=f"cuda:{self.device}")
            at = self._ws.data_ptr()
            self._ws_at = at + -at % 256
            self._ws_room = self._ws.numel() - -at % 256
        return self._ws_at

    def workspace(self, nbytes: int) -> torch.Tensor:
        off = self._scratch(nbytes) - self._ws.data_ptr()
        return self._ws[off:off + nbytes]

    # -- Section 3.2 --------------------------------------------------------------------------
    def channel_stats(self, calib: torch.Tensor, bins: int = 100):
        T, K = calib.shape
        ir = np.empty(K, dtype=np.float64)
        am = np.empty(K, dtype=np.float64)
        self._sync_stream()
        self._check(self._lib.esparse_channel_stats(self._h, _ptr(calib), T, K, _dtype_code(calib), bins,
                                                    ir.ctypes.data_as(C.c_void_p), am.ctypes.data_as(C.c_void_p)))
        return ir, am

    # -- Section 3.2 eq. 3 + Section 3.3 ------------------------------------------------------
    def prune(self, calib: Optional[torch.Tensor], W: torch.Tensor, opts: PruneOpts, *,
              score: Optional[np.ndarray] = None, want_retained: bool = False) -> PruneResult:
        N, K = W.shape
        dev = W.device
        perm = torch.empty(K, dtype=torch.int32, device=dev)
        mask = torch.empty((N, K), dtype=torch.uint8, device=dev)
        nblk = K // opts.block if (opts.block > 0 and K % opts.block == 0) else 0
        swaps = np.zeros(max(nblk, 1), dtype=np.int64)
        retained = C.c_double(0.0)
        co = opts._c()
        self._sync_stream()
        if score is None:
            T = calib.shape[0]
            assert calib.shape[1] == K and calib.dtype == W.dtype
            s_out = np.empty(K, dtype=np.float64)
            self._check(self._lib.esparse_prune(
                self._h, _ptr(calib), T, _ptr(W), N, K, _dtype_code(W), C.byref(co), _ptr(perm), _ptr(mask),
                s_out.ctypes.data_as(C.c_void_p), swaps.ctypes.data_as(C.c_void_p),
                C.cast(C.byref(retained), C.c_void_p) if want_retained else None))
        else:
            s_out = np.ascontiguousarray(score, dtype=np.float64)
            self._check(self._lib.esparse_prune_with_scores(
                self._h, s_out.ctypes.data_as(C.c_void_p), _ptr(W), N, K, _dtype_code(W), C.byref(co), _ptr(perm),
                _ptr(mask), swaps.ctypes.data_as(C.c_void_p),
                C.cast(C.byref(retained), C.c_void_p) if want_retained else None))
        return PruneResult(perm, mask, s_out, swaps[:nblk], retained.value if want_retained else None)

    # -- Section 4, step 1 --------------------------------------------------------------------
    def compress(self, W: torch.Tensor, mask: Optional[torch.Tensor], perm: Optional[torch.Tensor],
                 n_keep: int = 2, m_group: int = 4, *, canonical: bool = True, native: bool = True) -> Compressed:
        N, K = W.shape
        dt = _dtype_code(W)
        vb, mb, nb = _known_size(N, K, n_keep, m_group, dt)
        dev = W.device
        values = torch.empty((N, K * n_keep // m_group), dtype=W.dtype, device=dev) if canonical else None
        meta = torch.empty(mb, dtype=torch.uint8, device=dev) if canonical else None
        nat = torch.empty(nb, dtype=torch.uint8, device=dev) if native else None
        self._sync_stream()
        self._check(self._lib.esparse_compress(self._h, _ptr(W), _ptr(mask), _ptr(perm), N, K, dt, n_keep, m_group,
                                               _ptr(values), _ptr(meta), _ptr(nat)))
        return Compressed(values, meta, nat, N, K, n_keep, m_group, dt)

    # -- Section 4: products ------------------------------------------------------------------
    def spmm(self, X: torch.Tensor, comp: Compressed, perm: Optional[torch.Tensor], *, variant: int = -1,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
        M, K = X.shape
        assert K == comp.K and _dtype_code(X) == comp.dtype
        N = comp.N
        Y = out if out is not None else X.new_empty((M, N))
        nbytes = _known_workspace(M, N, K)
        ws = self._scratch(nbytes)
        self._sync_stream()
        rc = self._lib.esparse_spmm(self._h, X.data_ptr(), M, _ptr(comp.native), _ptr(perm), N, K, comp.dtype,
                                    comp.n_keep, comp.m_group, Y.data_ptr(), ws, nbytes, variant)
        if rc:
            self._check(rc)
        return Y

    def spmm_static(self, X: torch.Tensor, comp: Compressed, perm: Optional[torch.Tensor], *, variant: int = -1,
                    out: torch.Tensor) -> torch.Tensor:
        """esparse_spmm_static: the product with the library's own fixed scratch; nothing is allocated (the caller
        brings the output)."""
        M, K = X.shape
        assert K == comp.K and _dtype_code(X) == comp.dtype and tuple(out.shape) == (M, comp.N)
        self._sync_stream()
        self._check(self._lib.esparse_spmm_static(self._h, _ptr(X), M, _ptr(comp.native), _ptr(perm), comp.N, K, comp.dtype,
                                                  comp.n_keep, comp.m_group, _ptr(out), variant))
        return out

    def spmm_group(self, Xs, comps, perms, *, variant: int = -1, outs=None):
        """Products of one shape (same M, N, K, dtype, n:m) through one staging and one multiply launch
        where a decode kernel serves the shape; returns the list of outputs."""
        count = len(comps)
        assert len(Xs) == count and (perms is None or len(perms) == count)
        M, K = Xs[0].shape
        c0 = comps[0]
        N, X0, seen = c0.N, Xs[0], None
        for X, c in zip(Xs, comps):
            assert (c.N, c.K, c.dtype, c.n_keep, c.m_group) == (N, K, c0.dtype, c0.n_keep, c0.m_group)
            if X is not seen:
                assert tuple(X.shape) == (M, K) and _dtype_code(X) == c0.dtype
                seen = X
        if outs is None:
            outs = [X0.new_empty((M, N)) for _ in range(count)]
        nbytes = _known_group_workspace(count, M, N, K)
        ws = self._scratch(nbytes)
        self._sync_stream()
        rc = self._lib.esparse_spmm_group(self._h, count, _ptrs(Xs), M, _ptrs([c.native for c in comps]),
                                          _ptrs(perms) if perms is not None else None, N, K, c0.dtype, c0.n_keep, c0.m_group,
                                          _ptrs(outs), ws, nbytes, variant)
        if rc:
            self._check(rc)
        return outs

    def stage_activations_group(self, Xs, perms, comp0: Compressed, ws: torch.Tensor, *, variant: int = -1):
        count = len(Xs)
        M, K = Xs[0].shape
        ps = _ptrs(perms) if perms is not None else None
        self._sync_stream()
        self._check(self._lib.esparse_stage_activations_group(self._h, count, _ptrs(Xs), M, ps, comp0.N, K,
                                                              comp0.dtype, comp0.n_keep, comp0.m_group, _ptr(ws), ws.numel(), variant))

    def spmm_group_staged(self, M: int, comps, ws: torch.Tensor, outs, *, variant: int = -1):
        count = len(comps)
        c0 = comps[0]
        self._sync_stream()
        self._check(self._lib.esparse_spmm_group_staged(self._h, count, M, _ptrs([c.native for c in comps]), c0.N, c0.K,
                                                        c0.dtype, c0.n_keep, c0.m_group, _ptrs(outs), _ptr(ws),
                                                        ws.numel(), variant))
        return outs

    def dense_gemm_group(self, Xs, packed, N: int, *, variant: int = -1, outs=None):
        count = len(packed)
        M, K = Xs[0].shape
        if outs is None:
            outs = [torch.empty((M, N), dtype=Xs[0].dtype, device=Xs[0].device) for _ in range(count)]
        nbytes = _known_group_workspace(count, M, N, K)
        ws = self._scratch(nbytes)
        self._sync_stream()
        self._check(self._lib.esparse_dense_gemm_group(self._h, count, _ptrs(Xs), M, _ptrs(packed), N, K, _dtype_code(Xs[0]),
                                                       _ptrs(outs), ws, nbytes, variant))
        return outs

    def stage_activations(self, X: torch.Tensor, perm: Optional[torch.Tensor], N: int,
                          ws: Optional[torch.Tensor] = None) -> torch.Tensor:
        M, K = X.shape
        nbytes = _known_workspace(M, N, K)
        if ws is None:
            ws = self.workspace(nbytes)
        self._sync_stream()
        self._check(self._lib.esparse_stage_activations(self._h, _ptr(X), M, _ptr(perm), N, K, _dtype_code(X),
                                                        _ptr(ws), ws.numel()))
        return ws

    def spmm_staged(self, M: int, comp: Compressed, ws: torch.Tensor, Y: torch.Tensor, *, variant: int = -1):
        self._sync_stream()
        self._check(self._lib.esparse_spmm_staged(self._h, M, _ptr(comp.native), comp.N, comp.K, comp.dtype,
                                                  comp.n_keep, comp.m_group, _ptr(Y), _ptr(ws), ws.numel(), variant))
        return Y

    def dense_gemm_staged(self, M: int, packed: torch.Tensor, N: int, K: int, ws: torch.Tensor, Y: torch.Tensor, *,
                          variant: int = -1):
        self._sync_stream()
        self._check(self._lib.esparse_dense_gemm_staged(self._h, M, _ptr(packed), N, K, _dtype_code(Y), _ptr(Y),
                                                        _ptr(ws), ws.numel(), variant))
        return Y

    def dense_pack(self, W: torch.Tensor) -> torch.Tensor:
        N, K = W.shape
        packed = torch.empty(dense_packed_size(N, K), dtype=torch.uint8, device=W.device)
        self._sync_stream()
        self._check(self._lib.esparse_dense_pack(self._h, _ptr(W), N, K, _dtype_code(W), _ptr(packed)))
        return packed

    def dense_gemm(self, X: torch.Tensor, packed: torch.Tensor, N: int, *, variant: int = -1,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
        M, K = X.shape
        Y = out if out is not None else X.new_empty((M, N))
        nbytes = _known_workspace(M, N, K)
        ws = self._scratch(nbytes)
        self._sync_stream()
        self._check(self._lib.esparse_dense_gemm(self._h, X.data_ptr(), M, _ptr(packed), N, K, _dtype_code(X), Y.data_ptr(),
                                                 ws, nbytes, variant))
        return Y

    # -- Section 4, step 2 --------------------------------------------------------------------
    # -- Section 3.3 eq. 4 --------------------------------------------------------------------
    def output_error(self, Yref: torch.Tensor, Y: torch.Tensor):
        """(|| Yref - Y ||_F^2, || Yref ||_F^2) of two outputs of the same shape."""
        assert Yref.shape == Y.shape and Yref.dtype == Y.dtype and Yref.is_contiguous() and Y.is_contiguous()
        M, N = Yref.shape
        num, den = C.c_double(0.0), C.c_double(0.0)
        self._sync_stream()
        self._check(self._lib.esparse_output_error(self._h, _ptr(Yref), _ptr(Y), M, N, _dtype_code(Y),
                                                   C.cast(C.byref(num), C.c_void_p), C.cast(C.byref(den), C.c_void_p)))
        return num.value, den.value

    # -- measurement aid ------------------------------------------------------------------------
    def matrix_rate(self, sparse: bool = True, dtype: int = F16, random_operands: bool = True, mix: int = 0) -> float:
        """Effective TFLOP/s the matrix pipes sustain: mix 0 = operands held in registers, 1 = + a prefill stage's operand
        reads out of LDS, 2 = + its DMA, counted wait and barrier (L2-resident source)."""
        t = C.c_double(0.0)
        self._sync_stream()
        self._check(self._lib.esparse_matrix_rate(self._h, int(bool(sparse)), dtype, int(bool(random_operands)), mix, C.byref(t)))
        return t.value

    def read_rate(self, nbytes: int) -> float:
        """GB/s of a plain streaming read of nbytes per launch, cold (the launches walk through more than the caches hold)."""
        t = C.c_double(0.0)
        self._sync_stream()
        self._check(self._lib.esparse_read_rate(self._h, int(nbytes), C.byref(t)))
        return t.value

    def tune(self, M: int, N: int, K: int, dtype: int = F16, sparse=True):
        """sparse: False / 0 = dense, True / 1 = 2:4, 2 = 4:8."""
        best, ms = C.c_int(-1), C.c_float(0.0)
        self._sync_stream()
        self._check(self._lib.esparse_tune(self._h, M, N, K, dtype, int(sparse), C.byref(best), C.byref(ms)))
        return best.value, ms.value

    def tune_group(self, count: int, M: int, N: int, K: int, dtype: int = F16, sparse=True):
        """The same search for launches of `count` products of one shape (spmm_group, dense_gemm_group)."""
        best, ms = C.c_int(-1), C.c_float(0.0)
        self._sync_stream()
        self._check(self._lib.esparse_tune_group(self._h, count, M, N, K, dtype, int(sparse), C.byref(best), C.byref(ms)))
        return best.value, ms.value

    def tune_save(self, path: str):
        self._check(self._lib.esparse_tune_save(self._h, path.encode()))

    def tune_load(self, path: str):
        self._check(self._lib.esparse_tune_load(self._h, path.encode()))

    # -- microscaled numbers and the steps around a product -------------------------------------
    def _away(self, name: str, *tensors):
        where = ", ".join(str(t.device) for t in tensors)
        raise ValueError(f"{name}: a tensor is on {where}, the context on cuda:{self.device}")

    def _rows(self, name: str, t: torch.Tensor):
        """(rows, values of a row, values from row to row) of a matrix on the context's device whose rows are contiguous."""
        if t.get_device() != self.device:
            self._away(name, t)
        if t.dim() != 2:
            raise ValueError(f"{name}: {t.dim()} dimensions instead of two")
        R, K = t.shape
        if t.is_contiguous():
            return R, K, K
        if K > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}: the values of a row are {t.stride(1)} apart")
        if R > 1 and t.stride(0) < K:
            raise ValueError(f"{name}: rows overlap (stride {t.stride(0)} for {K} values)")
        return R, K, t.stride(0) if R > 1 else K

    def _check_mx(self, name: str, x: MX) -> int:
        """The number of rows; the tensors are on the context's device and of the format's shapes."""
        data, scales = x.data, x.scales
        if data.get_device() != self.device or scales.get_device() != self.device:
            self._away(name, data, scales)
        R, steps = data.shape[0], (x.K + 127) // 128
        if x.fmt not in (MX_FP4, MX_FP8):
            raise ValueError(f"{name}: format {x.fmt} is neither MX_FP4 nor MX_FP8")
        if data.shape != (R, steps * (64 if x.fmt == MX_FP4 else 128)) or scales.shape != (steps, R, 4):
            raise ValueError(f"{name}: data {tuple(data.shape)} and scales {tuple(scales.shape)} are not those of {R} rows of {x.K} channels")
        if data.dtype != torch.uint8 or scales.dtype != torch.uint8 or not data.is_contiguous() or not scales.is_contiguous():
            raise ValueError(f"{name}: data and scales are contiguous uint8 tensors")
        return R

    def _empty(self, rows: int, columns: int, dtype: torch.dtype) -> torch.Tensor:
        # (small calls wait for the host: 1.3 us with the strides given, 1.6 with new_empty, 1.2 with empty_like where a tensor of the shape is at hand)
        return _EMPTY((rows, columns), (columns, 1), dtype=dtype, device=self._on)

    def _empty_mx(self, R: int, K: int, fmt: int) -> MX:
        if fmt not in (MX_FP4, MX_FP8):
            raise ValueError(f"format {fmt} is neither MX_FP4 nor MX_FP8")
        steps = (K + 127) // 128
        return MX(self._empty(R, steps * (64 if fmt == MX_FP4 else 128), torch.uint8),
                  _EMPTY((steps, R, 4), (4 * R, 4, 1), dtype=torch.uint8, device=self._on), K, fmt)

    def mx_quantize(self, X: torch.Tensor, fmt: int) -> MX:
        """X[R, K] (f16, bf16, f32; rows may be apart) in microscaled 8 or 4 bits."""
        code, (R, K, ld) = _code(X.dtype, "mx_quantize", f32=True), self._rows("mx_quantize", X)
        out = self._empty_mx(R, K, fmt)
        self._sync_stream()
        rc = self._lib.esparse_mx_quantize(self._h, X.data_ptr(), R, K, ld, code, fmt, out.data.data_ptr(), out.scales.data_ptr())
        if rc:
            self._check(rc)
        return out

    def mx_dequantize(self, x: MX, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """The values [R, K] that x stands for."""
        code, R = _code(dtype, "mx_dequantize", f32=True), self._check_mx("mx_dequantize", x)
        out = self._empty(R, x.K, dtype)
        self._sync_stream()
        rc = self._lib.esparse_mx_dequantize(self._h, x.data.data_ptr(), x.scales.data_ptr(), R, x.K, x.fmt, code, out.data_ptr())
        if rc:
            self._check(rc)
        return out

    def mx_pack(self, w: MX) -> MXWeight:
        """Weights[N, K] in microscaled 4 bits, laid out once for mx_gemm."""
        N = self._check_mx("mx_pack", w)
        if w.fmt != MX_FP4:
            raise ValueError("mx_pack: weights are in 4 bits (MX_FP4)")
        packed = w.data.new_empty(mx_packed_size(N, w.K))
        self._sync_stream()
        self._check(self._lib.esparse_mx_pack(self._h, w.data.data_ptr(), w.scales.data_ptr(), N, w.K, packed.data_ptr()))
        return MXWeight(packed, N, w.K)

    def mx_gemm(self, X, w: MXWeight, *, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """X . W^T in `dtype` (f16, bf16 or f32).  X: an MX of 8 or 4 bits (dtype: bf16 if not given), or a 16-bit matrix whose rows may be apart
        (dtype: its own), with which the weights alone are in 4 bits."""
        packed, N = w.packed, w.N
        if isinstance(X, MX):
            M, K, act, code, ld, aligned = self._check_mx("mx_gemm", X), X.K, X.fmt, 0, 0, True
            x, scales, given = X.data.data_ptr(), X.scales.data_ptr(), torch.bfloat16
        else:
            given = X.dtype
            code, (M, K, ld), act = _code(given, "mx_gemm"), self._rows("mx_gemm", X), _ACT_16
            x, scales = X.data_ptr(), None
            aligned = not (ld % 8 or x % 16)
        if K != w.K:
            raise ValueError(f"mx_gemm: activations of {K} channels, weights of {w.K}")
        if packed.get_device() != self.device:
            self._away("mx_gemm", packed)
        if packed.dtype != torch.uint8 or packed.numel() != _known_mx_packed_size(N, K) or not packed.is_contiguous():
            raise ValueError(f"mx_gemm: packed is not the weights of {N} x {K}")
        if out is None:
            out = self._empty(M, N, dtype or given)
        elif out.get_device() != self.device:
            self._away("mx_gemm", out)
        elif out.shape != (M, N) or not out.is_contiguous() or (dtype is not None and out.dtype != dtype):
            raise ValueError(f"mx_gemm: out is not a contiguous [{M}, {N}] of the type asked for")
        out_code = _code(out.dtype, "mx_gemm", f32=True)
        nbytes = _known_mx_gemm_workspace(M, N, K, act, aligned)
        # a block of its own for each call: calls on several streams and captured graphs do not share it
        ws = packed.new_empty(nbytes) if nbytes else None
        self._sync_stream()
        rc = self._lib.esparse_mx_gemm(self._h, x, scales, M, ld, act, code, packed.data_ptr(), N, K, out_code, out.data_ptr(), _ptr(ws), nbytes)
        if rc:
            self._check(rc)
        return out

    def rms_norm(self, x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, *, residual: Optional[torch.Tensor] = None,
                 fmt: Optional[int] = None, sum_out: Optional[torch.Tensor] = None):
        """(y, h): h = x + residual (h is x itself where there is no residual), y = h weight / sqrt(mean(h^2) + eps), in the type of x
        (fmt None) or as an MX.  sum_out: where to write h; x or residual for an update in place."""
        dtype = x.dtype
        code, (R, K, ldx) = _code(dtype, "rms_norm"), self._rows("rms_norm", x)
        if weight.get_device() != self.device:
            self._away("rms_norm", weight)
        if weight.dtype != dtype or weight.shape != (K,) or not weight.is_contiguous():
            raise ValueError(f"rms_norm: weight is not a contiguous [{K}] of the type of x")
        r, ldr = None, 0
        if residual is not None:
            rows, channels, ldr = self._rows("rms_norm", residual)
            if residual.dtype != dtype or rows != R or channels != K:
                raise ValueError("rms_norm: residual is not of the shape and type of x")
            r = residual.data_ptr()
            if sum_out is None:
                sum_out = torch.empty_like(residual) if ldr == K else self._empty(R, K, dtype)
        if sum_out is not None:
            if sum_out.get_device() != self.device:
                self._away("rms_norm", sum_out)
            if sum_out.dtype != dtype or sum_out.shape != (R, K) or not sum_out.is_contiguous():
                raise ValueError("rms_norm: sum_out is not a contiguous tensor of the shape and type of x")
        h = None if sum_out is None else sum_out.data_ptr()
        if fmt is None:
            y = torch.empty_like(x) if ldx == K else self._empty(R, K, dtype)
            to = y.data_ptr(), 0, None, None
        else:
            y = self._empty_mx(R, K, fmt)
            to = None, fmt, y.data.data_ptr(), y.scales.data_ptr()
        self._sync_stream()
        rc = self._lib.esparse_rms_norm(self._h, x.data_ptr(), ldx, r, ldr, weight.data_ptr(), R, K, eps, code, h, *to)
        if rc:
            self._check(rc)
        return y, (x if sum_out is None else sum_out)

    def token_logprobs(self, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, *, top: int = 0) -> TokenLogprobs:
        """Per row of logits[R, V] (f16, bf16, f32; rows may be apart): ln p of tokens[R] (int64; below 0: none, gives 0), the entropy, and the
        `top` most probable tokens in order."""
        code, (R, V, ld) = _code(logits.dtype, "token_logprobs", f32=True), self._rows("token_logprobs", logits)
        nbytes = _known_logprobs_workspace(R, V, code, top)
        logprob = ids = lps = tok = lp = ip = tp = None
        if tokens is not None:
            if tokens.get_device() != self.device:
                self._away("token_logprobs", tokens)
            if tokens.dtype != torch.int64 or tokens.shape != (R,) or not tokens.is_contiguous():
                raise ValueError(f"token_logprobs: tokens is not a contiguous int64 [{R}]")
            logprob = _EMPTY((R,), (1,), dtype=torch.float32, device=self._on)
            tok, lp = tokens.data_ptr(), logprob.data_ptr()
        entropy = _EMPTY((R,), (1,), dtype=torch.float32, device=self._on)
        if top:
            ids, lps = self._empty(R, top, torch.int32), self._empty(R, top, torch.float32)
            ip, tp = ids.data_ptr(), lps.data_ptr()
        ws = _EMPTY((nbytes,), (1,), dtype=torch.uint8, device=self._on) if nbytes else None
        self._sync_stream()
        rc = self._lib.esparse_token_logprobs(self._h, logits.data_ptr(), R, V, ld, code, tok, top, lp, entropy.data_ptr(), ip, tp, _ptr(ws), nbytes)
        if rc:
            self._check(rc)
        return TokenLogprobs(logprob, entropy, ids, lps)
