"""MI355X-native emulated FP64 GEMM by Ozaki Scheme II: the published moduli's
or the all-byte moduli's (Sec. 5.1, candidate A) scale and results, computed
on int8 MFMA inside ozaki25_dgemm*; stages and stored planes on the set's own
planes, FP8 MFMA for the published moduli.

Python binding of ``libozaki25.so`` (the C ABI declared in
``include/ozaki25.h``).  Argument marshalling only: every step of the
computation runs in the library's HIP kernels.  PyTorch supplies device memory
and the current stream.  The binding fails loudly when the library has not
been built -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import re
import warnings

__all__ = [
    "Ozaki25Error", "lib", "library_path", "exported_symbols",
    "ozaki25_status_string", "ozaki25_num_moduli", "ozaki25_num_planes", "ozaki25_modulus",
    "ozaki25_scale_bits", "ozaki25_k_pad", "ozaki25_planes_bytes", "ozaki25_dgemm_workspace_size",
    "ozaki25_deconstruct", "ozaki25_residue_gemm", "ozaki25_reconstruct",
    "ozaki25_dgemm", "ozaki25_dgemm_sub", "ozaki25_dgemm_ex",
    "ozaki25_dgemm_planes_workspace_size", "ozaki25_dgemm_planes", "ozaki25_dgemm_noalloc",
    "ozaki25_accurate_exponents_workspace_size", "ozaki25_accurate_exponents",
    "ozaki25_dgemm_accurate_workspace_size", "ozaki25_dgemm_accurate",
    "ozaki25_grouped_matmul", "ozaki25_grouped_matmul_dx", "ozaki25_grouped_matmul_dw",
    "ozaki25_adapter_matmul_workspace_size", "ozaki25_adapter_matmul",
    "ozaki25_orthogonalise_workspace_size", "ozaki25_orthogonalise",
]

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libozaki25.so")
_HEADER = os.path.join(os.path.dirname(_PKG), "include", "ozaki25.h")

S12 = 0           # published moduli (own planes: FP8 limbs)
A15 = 1           # all-byte moduli (Sec. 5.1 candidate A; int8 planes)
RN = 0            # quantiser: round to nearest, ties to even (Ozaki-II-RN)
TZ = 1            # quantiser: toward zero (Ozaki-II-TZ)
NUM_MODULI = 12
NUM_PLANES = 30
NUM_MODULI_A15 = 15
K_ALIGN = 128
MAX_K = 4194304
MAX_N = 8388608
EXP_NONFINITE = -(2 ** 31)
NUM_STAGE_EVENTS = 5
NOALLOC_SCRATCH_BYTES = 128 << 20
BF16, F16, F32 = range(3)   # ozaki25_dtype
MAX_ROWS = 1 << 30          # limits of the 16-bit products
MAX_WIDTH = 1 << 22
MAX_LD = 1 << 32
MAX_GROUPS = 65536
MAX_RANK = 256
MAX_SIDE = 32768
MAX_STEPS = 64

SUCCESS, ERR_INVALID_VALUE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = range(5)


class Ozaki25Error(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {ozaki25_status_string(status)} (status {status})")
        self.status = status


_lib = None


def library_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is not built: run `python -m paper_2609_09095_amd.build`")
        L = ctypes.CDLL(_LIB_PATH)
        P, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
        f32 = ctypes.c_float
        sig = {
            "ozaki25_status_string": ([i32], ctypes.c_char_p),
            "ozaki25_num_moduli": ([i32], i32),
            "ozaki25_num_planes": ([i32], i32),
            "ozaki25_modulus": ([i32, i32], i64),
            "ozaki25_scale_bits": ([i64, i32], i32),
            "ozaki25_k_pad": ([i64], i64),
            "ozaki25_planes_bytes": ([i64, i64, i32], sz),
            "ozaki25_deconstruct": ([i32, i64, i64, P, i64, i32, i32, P, P, P], i32),
            "ozaki25_residue_gemm": ([i64, i64, i64, P, P, i32, P, P], i32),
            "ozaki25_reconstruct": ([i64, i64, P, P, P, i32, P, i64, i32, P], i32),
            "ozaki25_dgemm_workspace_size": ([i64, i64, i64, i32], sz),
            "ozaki25_dgemm": ([i64, i64, i64, P, i64, P, i64, P, i64, i32, P], i32),
            "ozaki25_dgemm_sub": ([i64, i64, i64, P, i64, P, i64, P, i64, i32, P], i32),
            "ozaki25_dgemm_ex": ([i64, i64, i64, P, i64, P, i64, P, i64, i32, i32, i32, P, sz, P, P], i32),
            "ozaki25_dgemm_planes_workspace_size": ([i64, i64, i64, i32], sz),
            "ozaki25_dgemm_planes": ([i64, i64, i64, P, P, P, P, P, i64, i32, i32, P, sz, P], i32),
            "ozaki25_dgemm_noalloc": ([i64, i64, i64, P, i64, P, i64, P, i64, i32, i32, i32, P], i32),
            "ozaki25_accurate_exponents_workspace_size": ([i64, i64, i64], sz),
            "ozaki25_accurate_exponents": ([i64, i64, i64, P, i64, P, i64, i32, P, P, P, sz, P], i32),
            "ozaki25_dgemm_accurate_workspace_size": ([i64, i64, i64, i32], sz),
            "ozaki25_dgemm_accurate": ([i64, i64, i64, P, i64, P, i64, P, i64, i32, i32, i32, P, sz, P, P],
                                       i32),
            "ozaki25_grouped_matmul": ([i64, i64, i64, i64, P, i64, P, i64, i64, P, P, i64, i32, P], i32),
            "ozaki25_grouped_matmul_dx": ([i64, i64, i64, i64, P, i64, P, i64, i64, P, P, i64, i32, P], i32),
            "ozaki25_adapter_matmul_workspace_size": ([i64, i64, i64, i64, i64], sz),
            "ozaki25_adapter_matmul": ([i64, i64, i64, i64, i64, P, i64, P, i64, P, P, i64, i64, P, i64, i64, P, P, i64,
                                        i32, P, sz, P], i32),
            "ozaki25_orthogonalise_workspace_size": ([i64, i64, i64], sz),
            "ozaki25_orthogonalise": ([i64, i64, i64, P, i64, i64, i32, P, i64, i64, i32, f32, f32, f32, f32, P, sz, P],
                                      i32),
            "ozaki25_grouped_matmul_dw": ([i64, i64, i64, i64, P, i64, P, i64, P, P, i64, i64, i32, i32, P], i32),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


def exported_symbols() -> list[str]:
    """Function names that include/ozaki25.h declares."""
    with open(_HEADER) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(ozaki25_[a-z0-9_]+)\s*\(", text)))


# ----------------------------------------------------------------- helpers
def _check(status: int, what: str):
    if status != SUCCESS:
        raise Ozaki25Error(status, what)


_torch = None     # torch, imported by the first call that handles tensors
_raw_stream = None  # () -> the current stream's handle


def _tensors():
    """torch; also picks the cheapest way to the current stream's handle (a
    Stream object costs a few microseconds, as much as a small product)."""
    global _torch, _raw_stream
    if _torch is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and dev is not None:
            _raw_stream = lambda: raw(dev())  # noqa: E731
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
        _torch = torch
    return _torch


# pointers and streams go to ctypes as plain integers (argtypes c_void_p)
def _stream(stream):
    if stream is None:
        _tensors()
        return _raw_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _on_gpu(ts):
    """Every tensor on one CUDA device (checked after the shapes and sizes,
    so that shape errors are reported first)."""
    dev, first = None, None
    for name, t in ts:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        d = t.get_device()
        if dev is None:
            dev, first = d, t
        elif d != dev:
            raise ValueError(f"{name} is on {t.device}, not on {first.device} like the other operands")


def _matrix(t, name, shape=None):
    """A 2-D float64 row-major matrix; returns (t, leading dimension)."""
    torch = _torch or _tensors()
    if not (isinstance(t, torch.Tensor) and t.dtype == torch.float64 and t.dim() == 2):
        raise ValueError(f"{name} must be a 2-D float64 tensor")
    rows, cols = t.shape
    if shape is not None and (rows, cols) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    s0, s1 = t.stride()
    if s1 != 1 and cols > 1:
        raise ValueError(f"{name} must be row-major (unit column stride)")
    if rows > 1 and s0 < cols:
        raise ValueError(f"{name} rows overlap (row stride below the row length)")
    return t, max(s0, cols, 1)


def _buffer(t, name, dtypes, numel):
    """A contiguous tensor of one of `dtypes` holding at least `numel` elements."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise ValueError(f"{name} must be a tensor of dtype {' or '.join(str(d) for d in dtypes)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, needs at least {numel}")
    return t


def _u8():
    import torch
    return (torch.uint8, torch.int8)


def _i32():
    import torch
    return (torch.int32,)


# ----------------------------------------------------------------- host-only
def ozaki25_status_string(status: int) -> str:
    return lib().ozaki25_status_string(status).decode()


def ozaki25_num_moduli(set: int = S12) -> int:
    return lib().ozaki25_num_moduli(set)


def ozaki25_num_planes(set: int = S12) -> int:
    return lib().ozaki25_num_planes(set)


def ozaki25_modulus(i: int, set: int = S12) -> int:
    return lib().ozaki25_modulus(set, i)


def ozaki25_scale_bits(k: int, set: int = S12) -> int:
    return lib().ozaki25_scale_bits(k, set)


def ozaki25_k_pad(k: int) -> int:
    return lib().ozaki25_k_pad(k)


def ozaki25_planes_bytes(vecs: int, k: int, set: int = S12) -> int:
    return lib().ozaki25_planes_bytes(vecs, k, set)


def ozaki25_dgemm_workspace_size(m: int, n: int, k: int, set: int = S12) -> int:
    return lib().ozaki25_dgemm_workspace_size(m, n, k, set)


# ----------------------------------------------------------------- stages
def ozaki25_deconstruct(side: int, X, planes=None, exps=None, set: int = S12, quantiser: int = RN,
                        stream=None):
    """side 0: X is A (rows); side 1: X is B (columns).  Returns (planes, exps):
    planes uint8 [k_pad/128][num_planes][vecs][128] (S12: limbs as OCP e4m3
    bytes; A15: int8 residues as two's complement bytes), exps int32 [vecs]."""
    import torch
    if side not in (0, 1):
        raise ValueError(f"side must be 0 (A) or 1 (B), not {side}")
    X, ldx = _matrix(X, "X")
    vecs, k = (X.shape[0], X.shape[1]) if side == 0 else (X.shape[1], X.shape[0])
    kp = ozaki25_k_pad(k)
    npl = ozaki25_num_planes(set)
    if npl < 0:
        raise ValueError(f"unknown modulus set {set}")
    if planes is None:
        planes = torch.empty((kp // K_ALIGN, npl, vecs, K_ALIGN), dtype=torch.uint8, device=X.device)
    if exps is None:
        exps = torch.empty((vecs,), dtype=torch.int32, device=X.device)
    _buffer(planes, "planes", _u8(), npl * vecs * kp)
    _buffer(exps, "exps", _i32(), vecs)
    _on_gpu([("X", X), ("planes", planes), ("exps", exps)])
    _check(lib().ozaki25_deconstruct(side, vecs, k, _ptr(X), ldx, set, quantiser, _ptr(planes),
                                     _ptr(exps), _stream(stream)), "ozaki25_deconstruct")
    return planes, exps


def ozaki25_residue_gemm(m: int, n: int, k: int, planesA, planesB, Cres=None, set: int = S12,
                         stream=None):
    """Centred per-modulus products, int32 [r][m][n]."""
    import torch
    r = ozaki25_num_moduli(set)
    if r < 0:
        raise ValueError(f"unknown modulus set {set}")
    if min(m, n, k) < 0:
        raise ValueError("negative dimension")
    _buffer(planesA, "planesA", _u8(), ozaki25_planes_bytes(m, k, set))
    _buffer(planesB, "planesB", _u8(), ozaki25_planes_bytes(n, k, set))
    if Cres is None:
        Cres = torch.empty((r, m, n), dtype=torch.int32, device=planesA.device)
    _buffer(Cres, "Cres", _i32(), r * m * n)
    _on_gpu([("planesA", planesA), ("planesB", planesB), ("Cres", Cres)])
    _check(lib().ozaki25_residue_gemm(m, n, k, _ptr(planesA), _ptr(planesB), set, _ptr(Cres),
                                      _stream(stream)), "ozaki25_residue_gemm")
    return Cres


def ozaki25_reconstruct(Cres, expsA, expsB, C=None, subtract: bool = False, set: int = S12,
                        stream=None):
    """C (m x n float64) from int32 residues [r][m][n] and the exponents."""
    import torch
    r = ozaki25_num_moduli(set)
    if r < 0:
        raise ValueError(f"unknown modulus set {set}")
    _buffer(expsA, "expsA", _i32(), 0)
    _buffer(expsB, "expsB", _i32(), 0)
    m, n = expsA.numel(), expsB.numel()
    _buffer(Cres, "Cres", _i32(), r * m * n)
    if C is None:
        C = torch.empty((m, n), dtype=torch.float64, device=Cres.device)
    C, ldc = _matrix(C, "C", (m, n))
    _on_gpu([("Cres", Cres), ("expsA", expsA), ("expsB", expsB), ("C", C)])
    _check(lib().ozaki25_reconstruct(m, n, _ptr(Cres), _ptr(expsA), _ptr(expsB), set, _ptr(C), ldc,
                                     1 if subtract else 0, _stream(stream)), "ozaki25_reconstruct")
    return C


# ----------------------------------------------------------------- GEMM
def _workspace(workspace):
    if workspace is None:
        return 0, 0
    _buffer(workspace, "workspace", _u8(), 0)
    return _ptr(workspace), workspace.numel()


def _events(stage_events):
    if stage_events is None:
        return None
    handles = []
    for e in stage_events:
        if not hasattr(e, "cuda_event") or not e.cuda_event:
            raise ValueError("stage events must be recorded torch.cuda.Event objects")
        handles.append(e.cuda_event)
    if len(handles) != NUM_STAGE_EVENTS:
        raise ValueError(f"need {NUM_STAGE_EVENTS} stage events")
    return ctypes.cast((ctypes.c_void_p * NUM_STAGE_EVENTS)(*handles), ctypes.c_void_p)


def _operands(A, B):
    A, lda = _matrix(A, "A")
    m, k = A.shape
    B, ldb = _matrix(B, "B")
    if B.shape[0] != k:
        raise ValueError(f"B has {B.shape[0]} rows, A has {k} columns")
    return A, lda, B, ldb, m, B.shape[1], k


def ozaki25_dgemm_ex(A, B, C, subtract: bool = False, workspace=None, stage_events=None,
                     set: int = S12, quantiser: int = RN, stream=None):
    A, lda, B, ldb, m, n, k = _operands(A, B)
    C, ldc = _matrix(C, "C", (m, n))
    ev = _events(stage_events)
    ws_ptr, ws_bytes = _workspace(workspace)
    _on_gpu([("A", A), ("B", B), ("C", C), ("workspace", workspace)])
    _check(lib().ozaki25_dgemm_ex(m, n, k, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, set, quantiser,
                                  1 if subtract else 0, ws_ptr, ws_bytes, ev, _stream(stream)),
           "ozaki25_dgemm_ex")
    return C


def ozaki25_accurate_exponents_workspace_size(m: int, n: int, k: int) -> int:
    return lib().ozaki25_accurate_exponents_workspace_size(m, n, k)


def ozaki25_accurate_exponents(A, B, expsA=None, expsB=None, set: int = S12, workspace=None,
                               stream=None):
    """The accurate mode's sigma (rows of A) and tau (columns of B): the
    magnitude digits, their int8 bound product and the shifts it admits.
    Returns (expsA, expsB), int32 CUDA tensors."""
    import torch
    A, lda, B, ldb, m, n, k = _operands(A, B)
    if expsA is None:
        expsA = torch.empty(m, dtype=torch.int32, device=A.device)
    if expsB is None:
        expsB = torch.empty(n, dtype=torch.int32, device=A.device)
    _buffer(expsA, "expsA", _i32(), m)
    _buffer(expsB, "expsB", _i32(), n)
    ws_ptr, ws_bytes = _workspace(workspace)
    _on_gpu([("A", A), ("B", B), ("expsA", expsA), ("expsB", expsB), ("workspace", workspace)])
    _check(lib().ozaki25_accurate_exponents(m, n, k, _ptr(A), lda, _ptr(B), ldb, set, _ptr(expsA),
                                            _ptr(expsB), ws_ptr, ws_bytes, _stream(stream)),
           "ozaki25_accurate_exponents")
    return expsA, expsB


def ozaki25_dgemm_accurate_workspace_size(m: int, n: int, k: int, set: int = S12) -> int:
    return lib().ozaki25_dgemm_accurate_workspace_size(m, n, k, set)


def ozaki25_dgemm_accurate(A, B, C=None, subtract: bool = False, workspace=None, stage_events=None,
                           set: int = S12, quantiser: int = RN, stream=None):
    """C = A B (or C -= A B) in the accurate mode: per-row and per-column
    shifts from the magnitude-bound product instead of the fixed t(k)."""
    import torch
    A, lda, B, ldb, m, n, k = _operands(A, B)
    if C is None:
        if subtract:
            raise ValueError("subtract needs C")
        C = torch.empty((m, n), dtype=torch.float64, device=A.device)
    C, ldc = _matrix(C, "C", (m, n))
    ev = _events(stage_events)
    ws_ptr, ws_bytes = _workspace(workspace)
    _on_gpu([("A", A), ("B", B), ("C", C), ("workspace", workspace)])
    _check(lib().ozaki25_dgemm_accurate(m, n, k, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, set, quantiser,
                                        1 if subtract else 0, ws_ptr, ws_bytes, ev, _stream(stream)),
           "ozaki25_dgemm_accurate")
    return C


def ozaki25_dgemm(A, B, C=None, set: int = S12, stream=None):
    """C = A B (float64, row-major CUDA tensors)."""
    import torch
    A, lda = _matrix(A, "A")
    m, k = A.shape
    B, ldb = _matrix(B, "B")
    if B.shape[0] != k:
        raise ValueError(f"B has {B.shape[0]} rows, A has {k} columns")
    n = B.shape[1]
    if C is None:
        C = torch.empty((m, n), dtype=torch.float64, device=A.device)
    C, ldc = _matrix(C, "C", (m, n))
    _on_gpu([("A", A), ("B", B), ("C", C)])
    _check(lib().ozaki25_dgemm(m, n, k, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, set,
                               _stream(stream)), "ozaki25_dgemm")
    return C


def ozaki25_dgemm_sub(A, B, C, set: int = S12, stream=None):
    """C <- C - A B in place."""
    A, lda = _matrix(A, "A")
    m, k = A.shape
    B, ldb = _matrix(B, "B")
    if B.shape[0] != k:
        raise ValueError(f"B has {B.shape[0]} rows, A has {k} columns")
    n = B.shape[1]
    C, ldc = _matrix(C, "C", (m, n))
    _on_gpu([("A", A), ("B", B), ("C", C)])
    _check(lib().ozaki25_dgemm_sub(m, n, k, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, set,
                                   _stream(stream)), "ozaki25_dgemm_sub")
    return C


def ozaki25_dgemm_planes_workspace_size(m: int, n: int, k: int, set: int = S12) -> int:
    return lib().ozaki25_dgemm_planes_workspace_size(m, n, k, set)


def ozaki25_dgemm_planes(k: int, planesA, expsA, planesB, expsB, C=None, subtract: bool = False,
                         workspace=None, set: int = S12, stream=None):
    """C = A B (or C -= A B) from stored planes (storage mode P): planes and
    exponents from ozaki25_deconstruct of A (side 0) and B (side 1) with this
    k and set.  m and n come from the exponent vectors."""
    import torch
    npl = ozaki25_num_planes(set)
    if npl < 0:
        raise ValueError(f"unknown modulus set {set}")
    if k < 0:
        raise ValueError("negative k")
    _buffer(expsA, "expsA", _i32(), 0)
    _buffer(expsB, "expsB", _i32(), 0)
    m, n = expsA.numel(), expsB.numel()
    _buffer(planesA, "planesA", _u8(), ozaki25_planes_bytes(m, k, set))
    _buffer(planesB, "planesB", _u8(), ozaki25_planes_bytes(n, k, set))
    if C is None:
        C = torch.empty((m, n), dtype=torch.float64, device=expsA.device)
    C, ldc = _matrix(C, "C", (m, n))
    ws_ptr, ws_bytes = _workspace(workspace)
    _on_gpu([("planesA", planesA), ("expsA", expsA), ("planesB", planesB), ("expsB", expsB), ("C", C),
             ("workspace", workspace)])
    _check(lib().ozaki25_dgemm_planes(m, n, k, _ptr(planesA), _ptr(expsA), _ptr(planesB), _ptr(expsB),
                                      _ptr(C), ldc, set, 1 if subtract else 0, ws_ptr, ws_bytes,
                                      _stream(stream)), "ozaki25_dgemm_planes")
    return C


def ozaki25_dgemm_noalloc(A, B, C=None, subtract: bool = False, set: int = S12, quantiser: int = RN,
                          stream=None):
    """C = A B (or C -= A B) with the library's static per-GPU workspace of
    NOALLOC_SCRATCH_BYTES: no device allocation.  Products whose workspace
    (ozaki25_dgemm_workspace_size) exceeds it raise Ozaki25Error with
    ERR_WORKSPACE.  Calls that overlap on one GPU race on that workspace."""
    import torch
    A, lda = _matrix(A, "A")
    m, k = A.shape
    B, ldb = _matrix(B, "B")
    if B.shape[0] != k:
        raise ValueError(f"B has {B.shape[0]} rows, A has {k} columns")
    n = B.shape[1]
    if C is None:
        if subtract:
            raise ValueError("subtract needs C")
        C = torch.empty((m, n), dtype=torch.float64, device=A.device)
    C, ldc = _matrix(C, "C", (m, n))
    _on_gpu([("A", A), ("B", B), ("C", C)])
    _check(lib().ozaki25_dgemm_noalloc(m, n, k, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, set, quantiser,
                                       1 if subtract else 0, _stream(stream)), "ozaki25_dgemm_noalloc")
    return C


# ----------------------------------------------------------------- 16-bit products
# A decode step's kernels take a few microseconds, as much as careless checks
# would: one look at each property of each tensor.  The calls are not recorded for
# gradients (ozaki25_grouped_matmul's are calls of their own); they warn where an
# input asks for one.
_HALF = None      # torch dtype -> ozaki25_dtype


def _half_types():
    global _HALF
    torch = _torch or _tensors()
    if _HALF is None:
        _HALF = {torch.bfloat16: BF16, torch.float16: F16}
    return _HALF


def _pitched(t, name, dims, types, shape=None):
    """A `dims`-dimensional tensor of one of `types`, elements of a row
    contiguous; returns (shape, row pitch, matrix pitch)."""
    if not (isinstance(t, _torch.Tensor) and t.dtype in types and t.dim() == dims):
        raise ValueError(f"{name} must be a {dims}-D tensor of dtype {' or '.join(str(d) for d in types)}")
    size = t.shape
    if shape is not None and size != shape:
        raise ValueError(f"{name} has shape {tuple(size)}, expected {tuple(shape)}")
    if dims == 3:
        count, rows, cols = size
    else:
        rows, cols = size
    if t.is_contiguous():
        ld = cols or 1
        return size, ld, rows * ld
    stride = t.stride()
    s0 = stride[-2]
    if stride[-1] != 1 and cols > 1:
        raise ValueError(f"{name} must be row-major (unit column stride)")
    if rows > 1 and s0 < cols:
        raise ValueError(f"{name} rows overlap (row stride below the row length)")
    ld = max(s0 if rows > 1 else cols, 1)
    return size, ld, stride[0] if dims == 3 and count > 1 else rows * ld


def _vector(t, name, dtype, count):
    """A contiguous vector of `count` elements of dtype."""
    if not (isinstance(t, _torch.Tensor) and t.dtype == dtype and t.dim() == 1 and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous 1-D {str(dtype).replace('torch.', '')} tensor")
    if t.numel() != count:
        raise ValueError(f"{name} holds {t.numel()} elements, expected {count}")


def _room(workspace):
    """Address and bytes of a workspace, 0 and 0 for none."""
    if workspace is None:
        return 0, 0
    if not (isinstance(workspace, _torch.Tensor) and workspace.dtype in (_torch.uint8, _torch.int8)
            and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous tensor of dtype torch.uint8 or torch.int8")
    return workspace.data_ptr(), workspace.numel()


def _together(first, names, *others):
    """Every tensor on the first one's GPU (checked after shapes and sizes)."""
    dev = first.get_device()
    for t in others:
        if t is not None and (dev < 0 or t.get_device() != dev):
            _on_gpu(zip(names, (first, *others)))
            return


def _unrecorded(what):
    """A warning, with an input that asks for a gradient, that none is recorded."""
    if _torch.is_grad_enabled():
        warnings.warn(f"{what} does not record gradients: its result is a constant to autograd, though an input requires "
                      "them (call it under torch.no_grad(), or in a torch.autograd.Function with the products that are "
                      "its gradients)", stacklevel=3)


def _new(like, shape, stream, dtype=None):
    """An output of the call beside `like`, of its dtype if none is given,
    allocated on the stream that writes it."""
    if stream is None or not like.is_cuda:
        return like.new_empty(shape, dtype=dtype)
    s = stream if hasattr(stream, "cuda_stream") else _torch.cuda.ExternalStream(int(stream), device=like.device)
    with _torch.cuda.stream(s):
        return like.new_empty(shape, dtype=dtype)


def ozaki25_grouped_matmul(X, W, ends, Y=None, stream=None):
    """Y[r] = X[r] W[g]^T for the rows r of group g.  X: rows x k, sorted by
    group; W: groups x n x k; ends: int32 [groups], one past each group's last
    row (read on the device).  bfloat16 or float16; rows past the last end are
    zeros.  Returns Y, rows x n."""
    types = _half_types()
    (rows, k), ldx, _ = _pitched(X, "X", 2, types)
    kind = (X.dtype,)
    (groups, n, kw), ldw, stride = _pitched(W, "W", 3, kind)
    if kw != k:
        raise ValueError(f"W has {kw} columns, X has {k}")
    _vector(ends, "ends", _torch.int32, groups)
    if X.requires_grad or W.requires_grad:
        _unrecorded("ozaki25_grouped_matmul")
    if Y is None:
        _together(X, ("X", "W", "ends"), W, ends)
        Y, ldy = _new(X, (rows, n), stream), n or 1
    else:
        _, ldy, _ = _pitched(Y, "Y", 2, kind, (rows, n))
        _together(X, ("X", "W", "ends", "Y"), W, ends, Y)
    _check(lib().ozaki25_grouped_matmul(rows, n, k, groups, X.data_ptr(), ldx, W.data_ptr(), ldw, stride,
                                        ends.data_ptr(), Y.data_ptr(), ldy, types[X.dtype], _stream(stream)),
           "ozaki25_grouped_matmul")
    return Y


def ozaki25_grouped_matmul_dx(dY, W, ends, dX=None, stream=None):
    """dX[r] = dY[r] W[g], the gradient of ozaki25_grouped_matmul's input.
    Returns dX, rows x k."""
    types = _half_types()
    (rows, n), lddy, _ = _pitched(dY, "dY", 2, types)
    kind = (dY.dtype,)
    (groups, nw, k), ldw, stride = _pitched(W, "W", 3, kind)
    if nw != n:
        raise ValueError(f"W has {nw} rows, dY has {n} columns")
    _vector(ends, "ends", _torch.int32, groups)
    if dY.requires_grad or W.requires_grad:
        _unrecorded("ozaki25_grouped_matmul_dx")
    if dX is None:
        _together(dY, ("dY", "W", "ends"), W, ends)
        dX, lddx = _new(dY, (rows, k), stream), k or 1
    else:
        _, lddx, _ = _pitched(dX, "dX", 2, kind, (rows, k))
        _together(dY, ("dY", "W", "ends", "dX"), W, ends, dX)
    _check(lib().ozaki25_grouped_matmul_dx(rows, n, k, groups, dY.data_ptr(), lddy, W.data_ptr(), ldw, stride,
                                           ends.data_ptr(), dX.data_ptr(), lddx, types[dY.dtype], _stream(stream)),
           "ozaki25_grouped_matmul_dx")
    return dX


def ozaki25_grouped_matmul_dw(dY, X, ends, dW=None, out_dtype=None, stream=None):
    """dW[g] = sum of dY[r]^T X[r] over the rows r of group g, the gradient of
    ozaki25_grouped_matmul's weights; zeros for an empty group.  out_dtype:
    the inputs' (the default) or float32.  Returns dW, groups x n x k."""
    types = _half_types()
    (rows, n), lddy, _ = _pitched(dY, "dY", 2, types)
    (rx, k), ldx, _ = _pitched(X, "X", 2, (dY.dtype,))
    if rx != rows:
        raise ValueError(f"X has {rx} rows, dY has {rows}")
    groups = ends.numel() if isinstance(ends, _torch.Tensor) else 0
    _vector(ends, "ends", _torch.int32, groups)
    if dY.requires_grad or X.requires_grad:
        _unrecorded("ozaki25_grouped_matmul_dw")
    if dW is None:
        dW = _new(dY, (groups, n, k), stream, out_dtype)
    elif out_dtype is not None and dW.dtype != out_dtype:
        raise ValueError(f"dW has dtype {dW.dtype}, out_dtype is {out_dtype}")
    _, lddw, stride = _pitched(dW, "dW", 3, (dY.dtype, _torch.float32), (groups, n, k))
    _together(dY, ("dY", "X", "ends", "dW"), X, ends, dW)
    out = F32 if dW.dtype == _torch.float32 else types[dY.dtype]
    _check(lib().ozaki25_grouped_matmul_dw(rows, n, k, groups, dY.data_ptr(), lddy, X.data_ptr(), ldx, ends.data_ptr(),
                                           dW.data_ptr(), lddw, stride, types[dY.dtype], out, _stream(stream)),
           "ozaki25_grouped_matmul_dw")
    return dW


def ozaki25_adapter_matmul_workspace_size(rows: int, n: int, k: int, adapters: int, rank: int) -> int:
    return lib().ozaki25_adapter_matmul_workspace_size(rows, n, k, adapters, rank)


def ozaki25_adapter_matmul(X, W, ids, A, B, scales=None, Y=None, workspace=None, stream=None):
    """Y[t] = X[t] W^T + scales[a] (X[t] A[a]^T) B[a]^T with a = ids[t]; rows
    whose id is outside [0, adapters) get the projection alone.  X: rows x k,
    W: n x k, ids: int32 [rows], A: adapters x rank x k, B: adapters x n x rank,
    bfloat16 or float16; scales: float32 [adapters].  Returns Y, rows x n."""
    types = _half_types()
    (rows, k), ldx, _ = _pitched(X, "X", 2, types)
    kind = (X.dtype,)
    (n, kw), ldw, _ = _pitched(W, "W", 2, kind)
    if kw != k:
        raise ValueError(f"W has {kw} columns, X has {k}")
    (adapters, rank, ka), lda, a_stride = _pitched(A, "A", 3, kind)
    if ka != k:
        raise ValueError(f"A has {ka} columns, X has {k}")
    _, ldb, b_stride = _pitched(B, "B", 3, kind, (adapters, n, rank))
    _vector(ids, "ids", _torch.int32, rows)
    if scales is not None:
        _vector(scales, "scales", _torch.float32, adapters)
    ws_ptr, ws_bytes = _room(workspace)
    if X.requires_grad or W.requires_grad or A.requires_grad or B.requires_grad or (
            scales is not None and scales.requires_grad):
        _unrecorded("ozaki25_adapter_matmul")
    if Y is None:
        _together(X, ("X", "W", "ids", "A", "B", "scales", "workspace"), W, ids, A, B, scales, workspace)
        Y, ldy = _new(X, (rows, n), stream), n or 1
    else:
        _, ldy, _ = _pitched(Y, "Y", 2, kind, (rows, n))
        _together(X, ("X", "W", "ids", "A", "B", "scales", "Y", "workspace"), W, ids, A, B, scales, Y, workspace)
    _check(lib().ozaki25_adapter_matmul(rows, n, k, adapters, rank, X.data_ptr(), ldx, W.data_ptr(), ldw,
                                        ids.data_ptr(), A.data_ptr(), lda, a_stride, B.data_ptr(), ldb, b_stride,
                                        _ptr(scales), Y.data_ptr(), ldy, types[X.dtype], ws_ptr, ws_bytes,
                                        _stream(stream)), "ozaki25_adapter_matmul")
    return Y


def ozaki25_orthogonalise_workspace_size(count: int, m: int, n: int) -> int:
    return lib().ozaki25_orthogonalise_workspace_size(count, m, n)


def ozaki25_orthogonalise(G, X=None, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                          workspace=None, stream=None):
    """The matrices of G (count x m x n, or one m x n; bfloat16, float16 or
    float32) orthogonalised by `steps` Newton-Schulz products.  Returns X,
    bfloat16, of G's shape."""
    types = _half_types()
    if not (isinstance(G, _torch.Tensor) and G.dim() in (2, 3)):
        raise ValueError("G must be a 2-D or 3-D tensor")
    dims = G.dim()
    size, ldg, g_stride = _pitched(G, "G", dims, (*types, _torch.float32))
    m, n = size[-2:]
    a, b, c = coefficients
    if G.requires_grad:
        _unrecorded("ozaki25_orthogonalise")
    if X is None:
        X = _new(G, size, stream, _torch.bfloat16)
    _, ldx, x_stride = _pitched(X, "X", dims, (_torch.bfloat16,), size)
    ws_ptr, ws_bytes = _room(workspace)
    _together(G, ("G", "X", "workspace"), X, workspace)
    _check(lib().ozaki25_orthogonalise(size[0] if dims == 3 else 1, m, n, G.data_ptr(), ldg, g_stride,
                                       types.get(G.dtype, F32), X.data_ptr(), ldx, x_stride, steps, a, b, c, eps,
                                       ws_ptr, ws_bytes, _stream(stream)), "ozaki25_orthogonalise")
    return X
