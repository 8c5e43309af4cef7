"""ctypes binding for libbakron.so -- argument marshalling only.

Every step of the solver runs in the library's HIP kernels; torch is used only
for device memory (``data_ptr()``), the current HIP stream and the range check of
pack_codes.  If the library has not been built, every call raises instead of falling
back to anything.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbakron.so")

BAKRON_OK, BAKRON_EINVAL, BAKRON_ENOTSPD, BAKRON_ENOMEM, BAKRON_EHIP = range(5)

EXPORTED = ("bakron_factor", "bakron_solve", "bakron_solve_debug", "bakron_factors_free",
            "bakron_status_string", "bakron_factors_error", "bakron_last_error",
            "bakron_factor_export", "bakron_profile_enable", "bakron_profile_read",
            "bakron_solve_check", "bakron_solve_antidiag", "bakron_gram",
            "bakron_sample_weights", "bakron_kron_factors", "bakron_mlp_local_factors",
            "bakron_mse_scales", "bakron_factor_blockdiag", "bakron_quadform_weights",
            "bakron_kron_factors_iter", "bakron_mlp_local_factors_iter", "bakron_solve_noalloc",
            "bakron_rmsnorm_quant", "bakron_pack_codes", "bakron_linear", "bakron_gated_mlp",
            "bakron_gated_mlp_backward", "bakron_token_logprobs", "bakron_token_logprobs_backward")

ALPHABETS = {"sym": 0, "asym": 1}

BAKRON_KFAC, BAKRON_SHAMPOO = 0, 1
STYLES = {"kfac": BAKRON_KFAC, "shampoo": BAKRON_SHAMPOO}

_lib = None


class BakronError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{status_string(status) if _lib else status}: {msg}")
        self.status = status


class _Quantizer(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("scale", ctypes.c_void_p), ("alphabet", ctypes.c_int32),
                ("group_size", ctypes.c_int32), ("col_scale", ctypes.c_void_p)]


class KernelStat(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double), ("launches", ctypes.c_int64), ("flops", ctypes.c_double),
                ("mfma_flops", ctypes.c_double)]

    def as_dict(self):
        return dict(ms=self.ms, launches=self.launches, flops=self.flops,
                    mfma_flops=self.mfma_flops)


def load(path: str = LIB_PATH):
    """Load libbakron.so (raises if it is missing: there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run __graft_entry__.build() first")
    lib = ctypes.CDLL(path)
    vp = ctypes.c_void_p
    lib.bakron_factor.restype = ctypes.c_int
    lib.bakron_factor.argtypes = [vp, ctypes.c_int64, vp, ctypes.c_int64, ctypes.c_float, vp,
                                  ctypes.POINTER(vp)]
    lib.bakron_solve.restype = ctypes.c_int
    lib.bakron_solve.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, vp, _Quantizer, vp, vp, vp]
    lib.bakron_solve_debug.restype = ctypes.c_int
    lib.bakron_solve_debug.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, vp, _Quantizer, vp, vp,
                                       vp, vp]
    lib.bakron_factors_free.restype = None
    lib.bakron_factors_free.argtypes = [vp]
    lib.bakron_status_string.restype = ctypes.c_char_p
    lib.bakron_status_string.argtypes = [ctypes.c_int]
    lib.bakron_factors_error.restype = ctypes.c_char_p
    lib.bakron_factors_error.argtypes = [vp]
    lib.bakron_last_error.restype = ctypes.c_char_p
    lib.bakron_last_error.argtypes = []
    lib.bakron_factor_export.restype = ctypes.c_int
    lib.bakron_factor_export.argtypes = [vp, ctypes.c_int, vp, vp]
    lib.bakron_profile_enable.restype = ctypes.c_int
    lib.bakron_profile_enable.argtypes = [vp, ctypes.c_int]
    lib.bakron_profile_read.restype = ctypes.c_int
    lib.bakron_profile_read.argtypes = [vp, ctypes.POINTER(KernelStat), ctypes.c_int]
    lib.bakron_solve_antidiag.restype = ctypes.c_int
    lib.bakron_solve_antidiag.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, vp, _Quantizer, vp, vp,
                                          vp, vp]
    lib.bakron_solve_noalloc.restype = ctypes.c_int
    lib.bakron_solve_noalloc.argtypes = [vp, ctypes.c_int64, ctypes.c_int64, vp, _Quantizer, vp, vp,
                                         vp]
    lib.bakron_solve_check.restype = ctypes.c_int
    lib.bakron_solve_check.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32)]
    i64, szp = ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)
    lib.bakron_mse_scales.restype = ctypes.c_int
    lib.bakron_mse_scales.argtypes = [vp, i64, i64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                      ctypes.c_int32, ctypes.c_double, vp, vp]
    lib.bakron_factor_blockdiag.restype = ctypes.c_int
    lib.bakron_factor_blockdiag.argtypes = [vp, i64, vp, i64, i64, ctypes.c_float, vp,
                                            ctypes.POINTER(vp)]
    lib.bakron_gram.restype = ctypes.c_int
    lib.bakron_gram.argtypes = [vp, i64, i64, vp, ctypes.c_float, vp, vp, vp, szp, vp]
    lib.bakron_sample_weights.restype = ctypes.c_int
    lib.bakron_sample_weights.argtypes = [vp, i64, i64, vp, vp, vp]
    lib.bakron_kron_factors.restype = ctypes.c_int
    lib.bakron_kron_factors.argtypes = [vp, vp, i64, i64, i64, ctypes.c_int32, vp, vp, vp, szp, vp]
    lib.bakron_quadform_weights.restype = ctypes.c_int
    lib.bakron_quadform_weights.argtypes = [vp, i64, i64, vp, vp, vp, szp, vp]
    lib.bakron_kron_factors_iter.restype = ctypes.c_int
    lib.bakron_kron_factors_iter.argtypes = [vp, vp, i64, i64, i64, ctypes.c_int32, vp, vp, vp,
                                             szp, vp]
    lib.bakron_mlp_local_factors_iter.restype = ctypes.c_int
    lib.bakron_mlp_local_factors_iter.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.c_int32, vp,
                                                  vp, vp, szp, vp]
    lib.bakron_mlp_local_factors.restype = ctypes.c_int
    lib.bakron_mlp_local_factors.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.c_int32, vp, vp, vp,
                                             szp, vp]
    i32, f32 = ctypes.c_int32, ctypes.c_float
    for name, args in (
            ("bakron_rmsnorm_quant", [vp, i64, vp, i64, i32, i64, i64, vp, f32, i32, vp, i64, vp, i64,
                                      vp, i64, vp, vp]),
            ("bakron_pack_codes", [vp, i64, i64, i32, vp, vp]),
            ("bakron_linear", [vp, i64, vp, i64, i64, vp, i32, i64, vp, i64, vp, i32, vp, i64, i32, vp,
                               i64, i32, vp, szp, vp]),
            ("bakron_gated_mlp", [vp, i64, i64, i64, vp, vp, i64, i64, i32, i32, vp, i64, vp, vp, vp,
                                  szp, vp]),
            ("bakron_gated_mlp_backward", [vp, i64, vp, i64, i64, i64, vp, vp, i64, i64, i32, i32, vp,
                                           i64, vp, vp, i64, vp, szp, vp]),
            ("bakron_token_logprobs", [vp, i64, i32, i64, i64, vp, i32, vp, vp, vp, vp, vp, vp, szp,
                                       vp]),
            ("bakron_token_logprobs_backward", [vp, i64, i32, i64, i64, vp, vp, vp, vp, vp, vp, i64,
                                                vp])):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = args
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().bakron_status_string(int(status)).decode()


def _on_its_device(fn):
    """The library launches on the current device: makes that of the first tensor the current
    one for the call."""
    @functools.wraps(fn)
    def call(*args, **kwargs):
        import torch
        first = args[0] if args else next(iter(kwargs.values()), None)
        device = getattr(first, "device", None)
        if getattr(device, "type", None) != "cuda" or device.index == torch.cuda.current_device():
            return fn(*args, **kwargs)
        with torch.cuda.device(device):
            return fn(*args, **kwargs)
    return call


def _stream(torch, device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _check_dev(t, name, dtype):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class Factors:
    """Owns a bakron_factors handle (normalised L^A, L^B in fp32 on the device)."""

    def __init__(self, handle: int, n: int, m: int | None, device):
        self._h = ctypes.c_void_p(handle)
        self.n = n
        self.m = m
        self.device = device

    @property
    def handle(self):
        return self._h

    def error(self) -> str:
        return load().bakron_factors_error(self._h).decode()

    @_on_its_device
    def export(self, which: str):
        """Dense fp32 copy of L^A ('A') or L^B ('B') for testing."""
        import torch
        d = self.n if which == "A" else (self.m or 0)
        out = torch.empty((max(d, 1), max(d, 1)), dtype=torch.float32, device=self.device)
        st = load().bakron_factor_export(self._h, 0 if which == "A" else 1,
                                         ctypes.c_void_p(out.data_ptr()),
                                         _stream(torch, self.device))
        if st != BAKRON_OK:
            raise BakronError(st, self.error())
        return out

    def profile(self, on: bool = True):
        """Enable/disable per-launch event timing (measurement hook)."""
        st = load().bakron_profile_enable(self._h, 1 if on else 0)
        if st != BAKRON_OK:
            raise BakronError(st, self.error())

    PROFILE_CLASSES = ("prep", "segment", "node")

    def _profile_stats(self):
        arr = (KernelStat * 4)()
        st = load().bakron_profile_read(self._h, arr, 4)
        if st != BAKRON_OK:
            raise BakronError(st, self.error())
        return [a.as_dict() for a in arr]

    def profile_read(self):
        """Per-class stats of the last profiled solve (stream must be synchronised)."""
        return dict(zip(self.PROFILE_CLASSES, self._profile_stats()))

    def profile_read_node_fp32(self):
        """The part of profile_read()["node"] that ran on fp32 MFMA (short nodes)."""
        return self._profile_stats()[3]

    @_on_its_device
    def check(self) -> bool:
        """True if every solve on this handle since the last check completed
        all of its ordered waits (synchronises the current stream; a give-up
        record is sticky on the device until this call clears it)."""
        import torch
        failed = ctypes.c_int32(0)
        st = load().bakron_solve_check(self._h, _stream(torch, self.device), ctypes.byref(failed))
        if st != BAKRON_OK:
            raise BakronError(st, self.error())
        return failed.value == 0

    def close(self):
        if self._h is not None and self._h.value:
            load().bakron_factors_free(self._h)
            self._h = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


@_on_its_device
def factor(A, B, damp: float) -> Factors:
    """bakron_factor(A, B, damp) on the current stream.  B=None means I."""
    import torch
    lib = load()
    _check_dev(A, "A", torch.float32)
    n = A.shape[0]
    if A.shape != (n, n):
        raise ValueError("A must be square")
    m = 0
    bptr = None
    if B is not None:
        _check_dev(B, "B", torch.float32)
        m = B.shape[0]
        if B.shape != (m, m):
            raise ValueError("B must be square")
        bptr = ctypes.c_void_p(B.data_ptr())
    h = ctypes.c_void_p(0)
    st = lib.bakron_factor(ctypes.c_void_p(A.data_ptr()), n, bptr, m, float(damp),
                           _stream(torch, A.device), ctypes.byref(h))
    if st != BAKRON_OK:
        raise BakronError(st, lib.bakron_last_error().decode())
    return Factors(h.value, n, m if B is not None else None, A.device)


def _quantizer(bits, scale, m, n, alphabet, group_size, col_scale):
    """bakron_quantizer for per-row (m) or per-(row, group) (m x ceil(n/g))
    scales, optional per-column factors, alphabet "sym" or "asym"."""
    import torch
    _check_dev(scale, "scale", torch.float32)
    g = int(group_size)
    if g < 0:
        raise ValueError("group_size must be >= 0")
    want = m * (-(-n // g)) if g > 0 else m
    if scale.numel() != want:
        raise ValueError(f"scale must have {want} entries")
    cp = None
    if col_scale is not None:
        _check_dev(col_scale, "col_scale", torch.float32)
        if col_scale.numel() != n:
            raise ValueError("col_scale must have n entries")
        cp = col_scale.data_ptr()
    if alphabet not in ALPHABETS:
        raise ValueError(f"alphabet must be one of {sorted(ALPHABETS)}")
    return _Quantizer(int(bits), ctypes.c_void_p(scale.data_ptr()).value, ALPHABETS[alphabet], g,
                      cp)


@_on_its_device
def solve(W, f: Factors, bits: int, scale, codes=None, V=None, pre=None, debug: bool = False,
          alphabet: str = "sym", group_size: int = 0, col_scale=None):
    """bakron_solve / bakron_solve_debug on the current stream.

    scale: m per-row scales, or m x ceil(n / group_size) with group_size > 0;
    col_scale: None or n per-column factors; alphabet "sym" or "asym".
    Returns (codes int8, V fp32) or (codes, V, pre) when debug=True.
    """
    import torch
    lib = load()
    _check_dev(W, "W", torch.float32)
    m, n = W.shape
    q = _quantizer(bits, scale, m, n, alphabet, group_size, col_scale)
    if codes is None:
        codes = torch.empty((m, n), dtype=torch.int8, device=W.device)
    if V is None:
        V = torch.empty((m, n), dtype=torch.float32, device=W.device)
    _check_dev(codes, "codes", torch.int8)
    _check_dev(V, "V", torch.float32)
    s = _stream(torch, W.device)
    if debug:
        if pre is None:
            pre = torch.empty((m, n), dtype=torch.float32, device=W.device)
        _check_dev(pre, "pre", torch.float32)
        st = lib.bakron_solve_debug(ctypes.c_void_p(W.data_ptr()), m, n, f.handle, q,
                                    ctypes.c_void_p(codes.data_ptr()), ctypes.c_void_p(V.data_ptr()),
                                    ctypes.c_void_p(pre.data_ptr()), s)
    else:
        st = lib.bakron_solve(ctypes.c_void_p(W.data_ptr()), m, n, f.handle, q,
                              ctypes.c_void_p(codes.data_ptr()), ctypes.c_void_p(V.data_ptr()), s)
    if st != BAKRON_OK:
        raise BakronError(st, f.error())
    return (codes, V, pre) if debug else (codes, V)


@_on_its_device
def solve_noalloc(W, f: Factors, bits: int, scale, codes=None, V=None, alphabet: str = "sym",
                  group_size: int = 0, col_scale=None):
    """bakron_solve_noalloc on the current stream: the solve with its workspace
    in the library's static per-device scratch (no device allocation).
    Quantiser arguments as :func:`solve`; codes and V are allocated here by
    torch only if not given.  Returns (codes int8, V fp32)."""
    import torch
    lib = load()
    _check_dev(W, "W", torch.float32)
    m, n = W.shape
    q = _quantizer(bits, scale, m, n, alphabet, group_size, col_scale)
    if codes is None:
        codes = torch.empty((m, n), dtype=torch.int8, device=W.device)
    if V is None:
        V = torch.empty((m, n), dtype=torch.float32, device=W.device)
    _check_dev(codes, "codes", torch.int8)
    _check_dev(V, "V", torch.float32)
    st = lib.bakron_solve_noalloc(ctypes.c_void_p(W.data_ptr()), m, n, f.handle, q,
                                  ctypes.c_void_p(codes.data_ptr()), ctypes.c_void_p(V.data_ptr()),
                                  _stream(torch, W.device))
    if st != BAKRON_OK:
        raise BakronError(st, f.error())
    return codes, V


@_on_its_device
def solve_antidiag(W, f: Factors, bits: int, scale, codes=None, V=None, pre=None,
                   alphabet: str = "sym", group_size: int = 0, col_scale=None):
    """bakron_solve_antidiag (BaKron-antidiagonal, Alg. 3) on the current stream.

    Quantiser arguments as :func:`solve`.
    Returns (codes int8, V fp32), or (codes, V, pre) when a pre buffer is given.
    """
    import torch
    lib = load()
    _check_dev(W, "W", torch.float32)
    m, n = W.shape
    q = _quantizer(bits, scale, m, n, alphabet, group_size, col_scale)
    if codes is None:
        codes = torch.empty((m, n), dtype=torch.int8, device=W.device)
    if V is None:
        V = torch.empty((m, n), dtype=torch.float32, device=W.device)
    _check_dev(codes, "codes", torch.int8)
    _check_dev(V, "V", torch.float32)
    if pre is not None:
        _check_dev(pre, "pre", torch.float32)
    st = lib.bakron_solve_antidiag(ctypes.c_void_p(W.data_ptr()), m, n, f.handle, q,
                                   ctypes.c_void_p(codes.data_ptr()), ctypes.c_void_p(V.data_ptr()),
                                   ctypes.c_void_p(pre.data_ptr() if pre is not None else None),
                                   _stream(torch, W.device))
    if st != BAKRON_OK:
        raise BakronError(st, f.error())
    return (codes, V) if pre is None else (codes, V, pre)


@_on_its_device
def factor_blockdiag(A, B_blocks, damp: float) -> Factors:
    """bakron_factor_blockdiag: B = blockdiag of B_blocks (nblocks x hb x hb)."""
    import torch
    lib = load()
    _check_dev(A, "A", torch.float32)
    _check_dev(B_blocks, "B_blocks", torch.float32)
    n = A.shape[0]
    if A.shape != (n, n) or B_blocks.dim() != 3 or B_blocks.shape[1] != B_blocks.shape[2]:
        raise ValueError("A must be n x n and B_blocks nblocks x hb x hb")
    nb, hb = B_blocks.shape[0], B_blocks.shape[1]
    h = ctypes.c_void_p(0)
    st = lib.bakron_factor_blockdiag(ctypes.c_void_p(A.data_ptr()), n,
                                     ctypes.c_void_p(B_blocks.data_ptr()), nb, hb, float(damp),
                                     _stream(torch, A.device), ctypes.byref(h))
    if st != BAKRON_OK:
        raise BakronError(st, lib.bakron_last_error().decode())
    return Factors(h.value, n, nb * hb, A.device)


@_on_its_device
def mse_scales(W, bits: int, alphabet: str = "sym", group_size: int = 0, grid: int = 100,
               maxshrink: float = 0.5):
    """bakron_mse_scales on the current stream: m scales, or m x ceil(n/g)."""
    import torch
    lib = load()
    _check_dev(W, "W", torch.float32)
    m, n = W.shape
    g = int(group_size)
    out = torch.empty((m, -(-n // g)) if g > 0 else (m,), dtype=torch.float32, device=W.device)
    st = lib.bakron_mse_scales(ctypes.c_void_p(W.data_ptr()), m, n, int(bits),
                               ALPHABETS[alphabet], g, int(grid), float(maxshrink),
                               ctypes.c_void_p(out.data_ptr()), _stream(torch, W.device))
    if st != BAKRON_OK:
        raise BakronError(st, lib.bakron_last_error().decode())
    return out


# ---------------------------------------------------------------- factor construction
def _ptr(t):
    return ctypes.c_void_p(t.data_ptr() if t is not None else None)


def _raise_last(st):
    if st != BAKRON_OK:
        raise BakronError(st, load().bakron_last_error().decode())


def _workspace(work, device):
    """Address and bytes of a caller's workspace: kernels write there, so it has to be
    memory of the device, without gaps."""
    if not work.is_cuda or work.device != device or not work.is_contiguous():
        raise ValueError(f"work must be contiguous on {device}")
    return work.data_ptr(), ctypes.c_size_t(work.numel() * work.element_size())


def _with_workspace(call, device):
    """Run a workspace-protocol entry point: query the size, allocate a torch
    buffer (256-byte aligned by the caching allocator), then call."""
    import torch
    need = ctypes.c_size_t(0)
    _raise_last(call(ctypes.c_void_p(None), ctypes.byref(need)))
    work = torch.empty(max(int(need.value), 256), dtype=torch.uint8, device=device)
    if work.data_ptr() % 256:
        raise RuntimeError("workspace is not 256-byte aligned")
    size = ctypes.c_size_t(work.numel())
    _raise_last(call(_ptr(work), ctypes.byref(size)))
    return work


@_on_its_device
def gram(X, w=None, s: float = 1.0, M=None, C=None, work=None):
    """bakron_gram: C = s * (X^T diag(w) X) (.) M on the current stream.
    X: N x d fp32; w: N or None; M: d x d or None (may be C itself)."""
    import torch
    lib = load()
    _check_dev(X, "X", torch.float32)
    N, d = X.shape
    for t, name, shape in ((w, "w", (N,)), (M, "M", (d, d))):
        if t is not None:
            _check_dev(t, name, torch.float32)
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} must have shape {shape}")
    if C is None:
        C = torch.empty((d, d), dtype=torch.float32, device=X.device)
    _check_dev(C, "C", torch.float32)
    if tuple(C.shape) != (d, d):
        raise ValueError("C must be d x d")
    st = _stream(torch, X.device)

    def call(wk, nbytes):
        return lib.bakron_gram(_ptr(X), N, d, _ptr(w), float(s), _ptr(M), _ptr(C), wk, nbytes, st)
    if work is None:
        _with_workspace(call, X.device)
    else:
        wp, size = _workspace(work, X.device)
        _raise_last(call(ctypes.c_void_p(wp), ctypes.byref(size)))
    return C


def gram_workspace_bytes(N: int, d: int) -> int:
    """Workspace bytes bakron_gram needs for an N x d sample matrix on the
    current device."""
    need = ctypes.c_size_t(0)
    _raise_last(load().bakron_gram(None, N, d, None, 1.0, None, None, None, ctypes.byref(need),
                                   None))
    return int(need.value)


@_on_its_device
def sample_weights(X, c=None, w=None):
    """bakron_sample_weights: w_k = sum_i c_i X_ki^2 on the current stream."""
    import torch
    lib = load()
    _check_dev(X, "X", torch.float32)
    N, d = X.shape
    if c is not None:
        _check_dev(c, "c", torch.float32)
        if c.numel() != d:
            raise ValueError("c must have d entries")
    if w is None:
        w = torch.empty((N,), dtype=torch.float32, device=X.device)
    _check_dev(w, "w", torch.float32)
    _raise_last(lib.bakron_sample_weights(_ptr(X), N, d, _ptr(c), _ptr(w),
                                          _stream(torch, X.device)))
    return w


@_on_its_device
def quadform_weights(X, M, w=None):
    """bakron_quadform_weights: w_k = x_k^T M x_k (M symmetric) on the current stream."""
    import torch
    lib = load()
    _check_dev(X, "X", torch.float32)
    _check_dev(M, "M", torch.float32)
    N, d = X.shape
    if tuple(M.shape) != (d, d):
        raise ValueError("M must be d x d")
    if w is None:
        w = torch.empty((N,), dtype=torch.float32, device=X.device)
    _check_dev(w, "w", torch.float32)
    st = _stream(torch, X.device)
    _with_workspace(lambda wk, nb: lib.bakron_quadform_weights(_ptr(X), N, d, _ptr(M), _ptr(w), wk,
                                                               nb, st), X.device)
    return w


@_on_its_device
def kron_factors(a, b, style: str = "kfac", iters: int = 1):
    """bakron_kron_factors (iters = 1) or bakron_kron_factors_iter (Shampoo
    with `iters` power steps): (A, B) of a global Hessian from paired vector
    samples a (N x n) and b (N x m) on the current stream."""
    import torch
    lib = load()
    _check_dev(a, "a", torch.float32)
    _check_dev(b, "b", torch.float32)
    N, n = a.shape
    if b.shape[0] != N:
        raise ValueError("a and b need the same number of samples")
    m = b.shape[1]
    A = torch.empty((n, n), dtype=torch.float32, device=a.device)
    B = torch.empty((m, m), dtype=torch.float32, device=a.device)
    st = _stream(torch, a.device)
    if iters != 1:
        if style != "shampoo":
            raise ValueError("power steps need style='shampoo'")
        _with_workspace(lambda wk, nb: lib.bakron_kron_factors_iter(
            _ptr(a), _ptr(b), N, n, m, int(iters), _ptr(A), _ptr(B), wk, nb, st), a.device)
        return A, B
    _with_workspace(lambda wk, nb: lib.bakron_kron_factors(_ptr(a), _ptr(b), N, n, m, STYLES[style],
                                                           _ptr(A), _ptr(B), wk, nb, st), a.device)
    return A, B


@_on_its_device
def mlp_local_factors(x, g, D, style: str = "kfac", iters: int = 1):
    """bakron_mlp_local_factors: (A, B) of the MLP-local Hessian from inputs x
    (N x dm), features g or f (N x dff) and W_down D (dm x dff)."""
    import torch
    lib = load()
    for t, name in ((x, "x"), (g, "g"), (D, "D")):
        _check_dev(t, name, torch.float32)
    N, dm = x.shape
    dff = g.shape[1]
    if g.shape[0] != N or tuple(D.shape) != (dm, dff):
        raise ValueError("shapes must be x: N x dm, g: N x dff, D: dm x dff")
    A = torch.empty((dm, dm), dtype=torch.float32, device=x.device)
    B = torch.empty((dff, dff), dtype=torch.float32, device=x.device)
    st = _stream(torch, x.device)
    if iters != 1:
        if style != "shampoo":
            raise ValueError("power steps need style='shampoo'")
        _with_workspace(lambda wk, nb: lib.bakron_mlp_local_factors_iter(
            _ptr(x), _ptr(g), _ptr(D), N, dm, dff, int(iters), _ptr(A), _ptr(B), wk, nb, st),
            x.device)
        return A, B
    _with_workspace(lambda wk, nb: lib.bakron_mlp_local_factors(_ptr(x), _ptr(g), _ptr(D), N, dm,
                                                                dff, STYLES[style], _ptr(A),
                                                                _ptr(B), wk, nb, st), x.device)
    return A, B


# ---------------------------------------------------------------- operators around a quantised layer
ACTS = {"none": 0, "silu": 1, "gelu": 2}
COMBINES = {"none": 0, "add": 1, "mul": 2}
PACK_COLUMNS = 128   # BAKRON_PACK_COLUMNS
_torch = None
_DTYPES = {}


def _import_torch():
    """torch, kept by name: small calls are bound by the host."""
    global _torch
    import torch
    _DTYPES.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
    _torch = torch
    return torch


def _dtype_code(dtype):
    """bakron_dtype of a torch dtype."""
    try:
        return _DTYPES[dtype]
    except KeyError:
        raise TypeError(f"dtype must be float32, float16 or bfloat16, got {dtype}") from None


def _rows_of(t, name, shape=None, dtype=None, device=None):
    """A 2-d tensor whose rows are contiguous (any distance between rows, none
    overlapping): its address and leading dimension."""
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}")
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != shape):
        raise ValueError(f"{name} must have shape {shape or '(rows, columns)'}, got {tuple(t.shape)}")
    rows, cols = t.shape
    ld, inner = t.stride()
    if cols > 1 and inner != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if rows <= 1:
        return t.data_ptr(), cols if rows == 0 or ld < cols else ld
    if ld < cols:
        raise ValueError(f"{name} must have rows that do not overlap")
    return t.data_ptr(), ld


def _vector(t, name, n, dtype, device):
    """A contiguous 1-d tensor of n entries, or None: its address."""
    if t is None:
        return None
    if not t.is_cuda or t.device != device:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with {n} entries")
    return t.data_ptr()


def _no_graph(name, instead, *tensors):
    """Refuses tensors whose gradients somebody expects: these calls record no graph, and a loss
    that came through one would silently have none."""
    for t in tensors:
        if t is not None and t.requires_grad and _torch.is_grad_enabled():
            raise RuntimeError(f"{name} records no graph for backward(): call it under torch.no_grad() or with "
                               f"detached tensors{instead}")


def _run(fn, args, device):
    """Call an operator on its tensors' device, on the current stream there (by its raw handle:
    small calls are bound by the host)."""
    torch = _torch or _import_torch()
    if torch._C._cuda_getDevice() != device.index:
        with torch.cuda.device(device):
            return _run(fn, args, device)
    _raise_last(fn(*args, torch._C._cuda_getCurrentRawStream(device.index)))


_work_sizes = {}


def _run_op(fn, args, device, work=None, key=None, maybe_none=True):
    """Call a workspace-protocol operator; allocates its workspace unless given.  `key`
    holds everything its size depends on, so that it is asked for once; maybe_none: it may
    need none, so try that first."""
    torch = _torch or _import_torch()
    if torch._C._cuda_getDevice() != device.index:
        with torch.cuda.device(device):
            return _run_op(fn, args, device, work, key, maybe_none)
    st = torch._C._cuda_getCurrentRawStream(device.index)
    if work is None:
        need = _work_sizes.get(key) if key is not None else None
        if need is None:
            size = ctypes.c_size_t(0)
            if key is None and maybe_none and fn(*args, 256, size, st) == BAKRON_OK:
                return   # needs none
            _raise_last(fn(*args, None, size, st))
            need = size.value
            if key is not None:
                _work_sizes[key] = need
        if need == 0:
            _raise_last(fn(*args, 256, ctypes.c_size_t(0), st))
            return
        work = torch.empty(need, dtype=torch.uint8, device=device)
    wp, size = _workspace(work, device)
    _raise_last(fn(*args, wp, size, st))


class NormQuant(NamedTuple):
    """What rmsnorm_quant returns: 8-bit rows (a view of rows padded to a multiple
    of 128 columns), their scales, and h and y where asked for."""
    q: object
    scale: object
    sum: object = None
    y: object = None


def rmsnorm_quant(x, weight=None, residual=None, eps: float = 1e-5, normalise: bool = True,
                  quantise: bool = True, with_sum: bool | None = None, with_y: bool = False,
                  sum_out=None):
    """bakron_rmsnorm_quant on the current stream: h = x + residual, y = weight *
    h / rms(h) (normalise=False: weight * h), q = rint(y / scale), scale = max |y| / 127
    per row.  x: T x d fp32, fp16 or bf16; weight: d fp32.  `sum` is returned where
    there is a residual, unless with_sum says otherwise; sum_out (e.g. residual
    itself) receives it.  Records no autograd graph."""
    torch = _torch or _import_torch()
    lib = load()
    _no_graph("rmsnorm_quant", "", x, weight, residual, sum_out)
    xp, ldx = _rows_of(x, "x")
    T, d = x.shape
    code = _dtype_code(x.dtype)
    dev = x.device
    rp, ldr = (None, d) if residual is None else _rows_of(residual, "residual", (T, d), x.dtype, dev)
    wp = _vector(weight, "weight", d, torch.float32, dev)
    if with_sum is None:
        with_sum = residual is not None or sum_out is not None
    hs = ys = q = scale = None
    sp = yp = qp = cp = None
    lds = ldy = ldq = d
    if with_sum:
        hs = torch.empty(T, d, dtype=x.dtype, device=dev) if sum_out is None else sum_out
        sp, lds = _rows_of(hs, "sum_out", (T, d), x.dtype, dev)
    if with_y:
        ys = torch.empty(T, d, dtype=x.dtype, device=dev)
        yp, ldy = ys.data_ptr(), d
    if quantise:
        ldq = -(-d // PACK_COLUMNS) * PACK_COLUMNS
        q = torch.empty(T, ldq, dtype=torch.int8, device=dev)
        scale = torch.empty(T, dtype=torch.float32, device=dev)
        qp, cp = q.data_ptr(), scale.data_ptr()
        if ldq != d:
            q = q[:, :d]
    _run(lib.bakron_rmsnorm_quant,
         (xp, ldx, rp, ldr, code, T, d, wp, float(eps), 1 if normalise else 0, sp, lds, yp, ldy, qp, ldq, cp), dev)
    return NormQuant(q, scale, hs, ys)


class PackedCodes(NamedTuple):
    """A layer's codes as bakron_linear reads them (bakron_pack_codes): `data` is
    m x bytes of a padded row, uint8; n columns of `width` bits."""
    data: object
    n: int
    width: int


def pack_codes(codes, width: int = 4, check: bool = True) -> PackedCodes:
    """bakron_pack_codes: lays out codes (m x n int8, e.g. of solve) once per layer.
    width 4 holds codes in [-8, 7]; others are refused, which waits for the codes (not
    with check=False, nor while the stream is being captured: their upper bits are then lost)."""
    torch = _torch or _import_torch()
    _check_dev(codes, "codes", torch.int8)
    if codes.dim() != 2:
        raise ValueError("codes must be m x n")
    if width == 4 and check and codes.numel() and not torch.cuda.is_current_stream_capturing():
        lo, hi = (int(v) for v in torch.aminmax(codes))
        if lo < -8 or hi > 7:
            raise ValueError(f"codes from {lo} to {hi} do not fit 4 bits: width 8 holds them")
    m, n = codes.shape
    padded = -(-n // PACK_COLUMNS) * PACK_COLUMNS
    data = torch.empty((m, padded * int(width) // 8), dtype=torch.uint8, device=codes.device)
    _run(load().bakron_pack_codes, (codes.data_ptr(), m, n, int(width), data.data_ptr()), codes.device)
    return PackedCodes(data, n, int(width))


def linear(q, q_scale, w: PackedCodes, scale, group_size: int = 0, bias=None, act: str = "none",
           other=None, combine: str | None = None, dtype=None, out=None, work=None):
    """bakron_linear on the current stream: act(q_scale * (q (scale * codes)^T) + bias),
    plus `other` (combine "add", the default where there is one) or times it ("mul").
    q, q_scale: as rmsnorm_quant returns them (T x n int8, T); scale: m, or m x
    ceil(n / group_size).  Returns T x m of dtype (default bf16).  Records no autograd graph."""
    torch = _torch or _import_torch()
    lib = load()
    _no_graph("linear", "", q_scale, scale, bias, other, out)
    qp, ldq = _rows_of(q, "q", None, torch.int8)
    dev = q.device
    T, n = q.shape
    if n != w.n:
        raise ValueError(f"q has {n} columns, the codes {w.n}")
    padded = -(-n // PACK_COLUMNS) * PACK_COLUMNS
    m, row_bytes = w.data.shape
    if row_bytes * 8 != padded * w.width or not w.data.is_contiguous() or w.data.device != dev or \
            w.data.dtype != torch.uint8:
        raise ValueError("w.data must be m x padded row bytes (uint8), contiguous, on q's device")
    if T <= 1:
        # the one row may be a view of any stride: what counts is what follows it
        ldq = padded
    if (q.storage_offset() + (T - 1) * ldq + padded if T else 0) > q.untyped_storage().nbytes():
        raise ValueError("q needs rows padded to a multiple of 128 columns (as rmsnorm_quant leaves them)")
    g = int(group_size)
    groups = -(-n // g) if g > 0 else 1
    # (the shape as well: as many scales in another order would give other products)
    if scale.dtype != torch.float32 or not scale.is_contiguous() or scale.device != dev or \
            (scale.shape != (m, groups) and (groups > 1 or scale.shape != (m,))):
        raise ValueError(f"scale must be contiguous fp32 of shape {(m, groups) if groups > 1 else (m,)} on {dev}")
    sp = _vector(q_scale, "q_scale", T, torch.float32, dev)
    if out is None:
        out = torch.empty(T, m, dtype=torch.bfloat16 if dtype is None else dtype, device=dev)
    yp, ldy = _rows_of(out, "out", (T, m), dtype, dev)
    code = _dtype_code(out.dtype)
    bp = _vector(bias, "bias", m, out.dtype, dev)
    op, ldo = (None, m) if other is None else _rows_of(other, "other", (T, m), out.dtype, dev)
    if combine is None:
        combine = "none" if other is None else "add"
    _run_op(lib.bakron_linear,
            (qp, ldq, sp, T, n, w.data.data_ptr(), w.width, m, scale.data_ptr(), g, bp, ACTS[act], op,
             ldo, COMBINES[combine], yp, ldy, code), dev, work)
    return out


def _mlp_operands(x, w_gate, w_up):
    xp, ldx = _rows_of(x, "x")
    T, d = x.shape
    gp, ldw = _rows_of(w_gate, "w_gate", None, x.dtype, x.device)
    f = w_gate.shape[0]
    up, ldu = _rows_of(w_up, "w_up", (f, d), x.dtype, x.device)
    if f <= 1:
        ldw = ldu = d   # (one row has no next one)
    if w_gate.shape[1] != d or ldu != ldw:
        raise ValueError("w_gate and w_up must be f x d with the same distance between rows")
    return xp, ldx, T, d, gp, up, ldw, f, _dtype_code(x.dtype)


class MlpFeatures(NamedTuple):
    """What gated_mlp returns with features=True: the output and the fp32 features
    that mlp_local_factors takes for W_up and for W_gate."""
    h: object
    up: object
    gate: object


def gated_mlp(x, w_gate, w_up, act: str = "silu", features: bool = False, out=None, work=None):
    """bakron_gated_mlp on the current stream: act(x w_gate^T) * (x w_up^T) in one
    kernel.  x: T x d, w_gate, w_up: f x d, all fp16 or all bf16.  features=True
    also returns act(G) and act'(G) * U in fp32.  Records no autograd graph: the gradients
    come from gated_mlp_backward."""
    torch = _torch or _import_torch()
    lib = load()
    _no_graph("gated_mlp", " and take the gradients from gated_mlp_backward", x, w_gate, w_up, out)
    xp, ldx, T, d, gp, up, ldw, f, code = _mlp_operands(x, w_gate, w_up)
    if out is None:
        out = torch.empty(T, f, dtype=x.dtype, device=x.device)
    hp, ldh = _rows_of(out, "out", (T, f), x.dtype, x.device)
    fu = fg = None
    if features:
        fu, fg = (torch.empty(T, f, dtype=torch.float32, device=x.device) for _ in range(2))
    _run_op(lib.bakron_gated_mlp,
            (xp, ldx, T, d, gp, up, ldw, f, code, ACTS[act], hp, ldh,
             fu.data_ptr() if features else None, fg.data_ptr() if features else None), x.device, work)
    return MlpFeatures(out, fu, fg) if features else out


def gated_mlp_backward(dh, x, w_gate, w_up, act: str = "silu", need_dx: bool = True,
                       need_dw: bool = True, work=None):
    """bakron_gated_mlp_backward: (dx, dw_gate, dw_up) from dh, the gradient with
    respect to gated_mlp's output; None for what is not needed."""
    torch = _torch or _import_torch()
    lib = load()
    xp, ldx, T, d, gp, up, ldw, f, code = _mlp_operands(x, w_gate, w_up)
    hp, ldh = _rows_of(dh, "dh", (T, f), x.dtype, x.device)
    dx = torch.empty(T, d, dtype=x.dtype, device=x.device) if need_dx else None
    dg, du = (torch.empty(f, d, dtype=x.dtype, device=x.device) if need_dw else None for _ in range(2))
    _run_op(lib.bakron_gated_mlp_backward,
            (hp, ldh, xp, ldx, T, d, gp, up, ldw, f, code, ACTS[act], dx.data_ptr() if need_dx else None,
             d, dg.data_ptr() if need_dw else None, du.data_ptr() if need_dw else None, d), x.device, work,
            maybe_none=False)
    return dx, dg, du


class TokenLogprobs(NamedTuple):
    """What token_logprobs returns (logprob None without targets, the top
    alternatives None without `top`)."""
    logprob: object
    entropy: object
    lse: object
    top_logprob: object = None
    top_index: object = None


def token_logprobs(logits, target=None, top: int = 0, work=None) -> TokenLogprobs:
    """bakron_token_logprobs on the current stream.  logits: T x V fp32, fp16 or
    bf16; target: T int64 (outside [0, V): ignored, 0) or None; top: number of
    alternatives, at most 32.  Records no autograd graph: the gradients come from
    token_logprobs_backward."""
    torch = _torch or _import_torch()
    lib = load()
    _no_graph("token_logprobs", " and take the gradients from token_logprobs_backward", logits)
    zp, ld = _rows_of(logits, "logits")
    T, V = logits.shape
    dev = logits.device
    tp = _vector(target, "target", T, torch.int64, dev)
    stats = torch.empty(3, T, dtype=torch.float32, device=dev)
    logprob, entropy, lse = stats.unbind(0)
    top = int(top)
    tl = ti = None
    if top > 0:
        tl = torch.empty(T, top, dtype=torch.float32, device=dev)
        ti = torch.empty(T, top, dtype=torch.int64, device=dev)
    _run_op(lib.bakron_token_logprobs,
            (zp, ld, _dtype_code(logits.dtype), T, V, tp, top, None if tp is None else logprob.data_ptr(),
             entropy.data_ptr(), lse.data_ptr(), None if tl is None else tl.data_ptr(),
             None if ti is None else ti.data_ptr()), dev, work,
            ("token_logprobs", T, V, top, logits.dtype))
    return TokenLogprobs(None if tp is None else logprob, entropy, lse, tl, ti)


def token_logprobs_backward(logits, target, lse, entropy=None, g_logprob=None, g_entropy=None, out=None):
    """bakron_token_logprobs_backward: the gradient with respect to the logits, T x V
    in their dtype (out may be logits itself), from the gradients with respect to
    token_logprobs' logprob and entropy (None for 0)."""
    torch = _torch or _import_torch()
    lib = load()
    zp, ld = _rows_of(logits, "logits")
    T, V = logits.shape
    dev = logits.device
    if out is None:
        out = torch.empty(T, V, dtype=logits.dtype, device=dev)
    dp, ldd = _rows_of(out, "out", (T, V), logits.dtype, dev)
    f32 = torch.float32
    _run(lib.bakron_token_logprobs_backward,
         (zp, ld, _dtype_code(logits.dtype), T, V, _vector(target, "target", T, torch.int64, dev),
          _vector(lse, "lse", T, f32, dev), _vector(entropy, "entropy", T, f32, dev),
          _vector(g_logprob, "g_logprob", T, f32, dev), _vector(g_entropy, "g_entropy", T, f32, dev), dp, ldd), dev)
    return out
