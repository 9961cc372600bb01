"""Python binding of the MOSAIC C ABI (include/mosaic.h).

Each function has the name of the ABI entry point it calls and only marshals
arguments: torch tensors (device memory, on the current HIP stream) become
pointers, leading dimensions and sizes. All arithmetic runs in the HIP
kernels of libmosaic.so. The functions of an online call hand their arguments
to _binding.so first (csrc/binding.cpp), which checks and converts a
well-formed call natively; it declines any other, and the Python code below
then handles it or says what is wrong with it.

Digit-layout matrices are ``Digits`` views: an int8 tensor of shape
(rows, pitch) plus a column offset (a multiple of 64), so several factors can
share one buffer side by side.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import List, Optional, Sequence, Tuple

import torch

from . import _lib

DIST_ZERO, DIST_UNIFORM, DIST_DGAUSS, DIST_SPARSE, DIST_WEIGHT = 0, 1, 2, 3, 4
DT_I8, DT_I16, DT_I32, DT_U32 = 0, 1, 2, 3
STATUS_OK, STATUS_INVALID_ARG, STATUS_UNSUPPORTED, STATUS_HIP = 0, -1, -2, -3
_TORCH_DT = {torch.int8: DT_I8, torch.int16: DT_I16, torch.int32: DT_I32}


class MosaicError(RuntimeError):
    def __init__(self, status: int, name: str):
        msg = _lib.load().mosaic_last_error_message().decode(errors="replace")
        super().__init__(f"{name} failed with status {status}: {msg}")
        self.status = status


def _check(status: int, name: str) -> None:
    if status != 0:
        raise MosaicError(status, name)


# Entry points that _binding.so calls, in the order it expects.
_BOUND = ("mosaic_sample", "mosaic_mask", "mosaic_masked_matmul", "mosaic_integrity_check", "mosaic_unmask",
          "mosaic_unmask_words", "mosaic_rotate_quantize_mask", "mosaic_sparse_stream_gather_rows_terms",
          "mosaic_sparse_gather_cols_terms", "mosaic_sparse_gather_cols", "mosaic_hadamard_rotate", "mosaic_quantize_rows",
          "mosaic_cache_append", "mosaic_cache_attend_workspace", "mosaic_cache_attend",
          "mosaic_cache_evict_workspace", "mosaic_cache_evict")
_b = None


def _native():
    """The native marshalling, bound to the loaded library on first use."""
    global _b
    if _b is None:
        lib = _lib.load()
        why = _lib.binding_stale_reason()
        if why is not None:
            raise RuntimeError(f"_binding.so is not usable ({why}): run `python -m paper_2607_29221_amd.build`")
        from . import _binding
        _binding.bind(tuple(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _BOUND),
                      torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, _lib.MosaicRng)
        _b = _binding
    return _b


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def padded_k(k: int) -> int:
    return 64 * ((k + 63) // 64)


# Host-side shape checks before any launch: the C ABI sees only pointers and
# sizes, so a tensor smaller than the sizes passed would be read or written
# past its end on the GPU. These raise ValueError instead.
def _need(t: Optional[torch.Tensor], rows: int, cols: int, name: str, dtypes=None, optional: bool = True) -> None:
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if rows == 0 or cols == 0:
        return
    if t.dim() == 1:
        if rows * cols > t.numel() or (rows > 1 and cols > 1):
            raise ValueError(f"{name} holds {t.numel()} elements, needs {rows} x {cols}")
        return
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    if t.shape[0] < rows or t.shape[1] < cols:
        raise ValueError(f"{name} is {tuple(t.shape)}, needs at least ({rows}, {cols})")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")


def _need_dig(d: Optional["Digits"], rows: int, cols: int, name: str, optional: bool = True) -> None:
    if d is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if not d.buf.is_cuda or d.buf.dtype != torch.int8 or d.buf.dim() != 2 or d.buf.stride(1) != 1:
        raise ValueError(f"{name} must be a row-contiguous int8 device matrix")
    if rows == 0 or cols == 0:
        return
    if d.rows < rows or d.col0 % 64 or 4 * (d.col0 + padded_k(cols)) > d.pitch:
        raise ValueError(f"{name} ({d.rows} rows, pitch {d.pitch}, column {d.col0}) cannot hold {rows} x {cols} digits")


_INT = (torch.int32,)


@dataclass
class Digits:
    """rows x cols ring matrix in digit layout, at column ``col0`` of ``buf``."""
    buf: torch.Tensor          # int8, (rows, pitch)
    cols: int
    col0: int = 0

    @property
    def rows(self) -> int:
        return self.buf.shape[0]

    @property
    def pitch(self) -> int:
        return self.buf.shape[1]

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr() + 4 * self.col0

    @staticmethod
    def empty(rows: int, cols: int, device="cuda") -> "Digits":
        return Digits(torch.empty((rows, 4 * padded_k(cols)), dtype=torch.int8, device=device), cols)

    @staticmethod
    def concat(rows: int, cols: Sequence[int], device="cuda") -> List["Digits"]:
        """Factors side by side in one buffer (each padded to 64 columns)."""
        total = sum(padded_k(c) for c in cols)
        buf = torch.empty((rows, 4 * max(total, 64)), dtype=torch.int8, device=device)
        out, off = [], 0
        for c in cols:
            out.append(Digits(buf, c, off))
            off += padded_k(c)
        return out

    def whole(self, cols: int) -> "Digits":
        """The full buffer seen as one matrix of ``cols`` columns from column 0."""
        return Digits(self.buf, cols, 0)


def rng(seed: int, stream: int, instance: int, dist: int, sigma: float = 0.5, bound: int = 4,
        log2_inv_density: int = 6, transposed: bool = False, row_weight: int = 0) -> _lib.MosaicRng:
    return _lib.MosaicRng(seed=seed & 0xFFFFFFFFFFFFFFFF, stream=stream, instance=instance, dist=dist,
                          bound=bound, sigma=sigma, log2_inv_density=log2_inv_density,
                          transposed=1 if transposed else 0, row_weight=row_weight)


def mosaic_abi_version() -> int:
    return _lib.load().mosaic_abi_version()


def mosaic_dgauss_thresholds(sigma: float, bound: int) -> List[int]:
    arr = (ctypes.c_uint64 * max(2 * bound, 1))()
    _check(_lib.load().mosaic_dgauss_thresholds(sigma, bound, arr), "mosaic_dgauss_thresholds")
    return [int(arr[i]) for i in range(2 * bound)]


def mosaic_sample(r: _lib.MosaicRng, rows: int, cols: int, out: Optional[torch.Tensor] = None,
                  out_dig: Optional[Digits] = None) -> None:
    st = (_b or _native()).sample(r, rows, cols, out, out_dig)
    if st is not None:
        return _check(st, "mosaic_sample")
    _need(out, rows, cols, "out", _INT)
    _need_dig(out_dig, rows, cols, "out_dig")
    ldo = out.stride(0) if out is not None else 0
    _check(_lib.load().mosaic_sample(ctypes.byref(r), rows, cols, _ptr(out), ldo,
                                     out_dig.ptr if out_dig else None, out_dig.pitch if out_dig else 0,
                                     _stream()), "mosaic_sample")


def mosaic_mask(x: Optional[torch.Tensor], u: Optional[torch.Tensor], noise: Optional[_lib.MosaicRng],
                rows: int, cols: int, out: Optional[torch.Tensor] = None,
                out_dig: Optional[Digits] = None, x_transposed: bool = False) -> None:
    """out = x + u + noise (mod 2^32). ``x_transposed`` reads x[j, i] for
    element (i, j) (x then has shape (cols, rows))."""
    st = (_b or _native()).mask(x, u, noise, rows, cols, out, out_dig, x_transposed)
    if st is not None:
        return _check(st, "mosaic_mask")
    if x is not None:
        if x.dtype not in _TORCH_DT or not x.is_cuda or x.dim() != 2:
            raise ValueError("x must be an int8/int16/int32 device matrix")
        xr, xc = (cols, rows) if x_transposed else (rows, cols)
        if x.shape[0] < xr or x.shape[1] < xc:
            raise ValueError(f"x is {tuple(x.shape)}, needs at least ({xr}, {xc})")
        dt = _TORCH_DT[x.dtype]   # int32 and uint32 embed identically into the ring
        rs, cs = (x.stride(1), x.stride(0)) if x_transposed else (x.stride(0), x.stride(1))
    else:
        dt, rs, cs = DT_U32, 0, 0
    _need(u, rows, cols, "u", _INT)
    _need(out, rows, cols, "out", _INT)
    _need_dig(out_dig, rows, cols, "out_dig")
    ldu = u.stride(0) if u is not None else 0
    ldo = out.stride(0) if out is not None else 0
    _check(_lib.load().mosaic_mask(_ptr(x), dt, rs, cs, _ptr(u), ldu,
                                   ctypes.byref(noise) if noise is not None else None, rows, cols,
                                   _ptr(out), ldo, out_dig.ptr if out_dig else None,
                                   out_dig.pitch if out_dig else 0, _stream()), "mosaic_mask")


def mosaic_masked_matmul(a: Digits, b: Digits, M: int, N: int, K: int, c: torch.Tensor) -> None:
    """c[:M, :N] = A B^T over Z_{2^32} (c is an int32 tensor holding ring words)."""
    st = (_b or _native()).masked_matmul(a, b, M, N, K, c)
    if st is not None:
        return _check(st, "mosaic_masked_matmul")
    _need_dig(a, M, K, "a", optional=False)
    _need_dig(b, N, K, "b", optional=False)
    _need(c, M, N, "c", _INT, optional=False)
    _check(_lib.load().mosaic_masked_matmul(a.ptr, a.pitch, b.ptr, b.pitch, M, N, K, c.data_ptr(),
                                            c.stride(0), _stream()), "mosaic_masked_matmul")


def mosaic_masked_matmul_words(a: Digits, b: torch.Tensor, M: int, N: int, K: int, c: torch.Tensor,
                               accumulate: bool = False) -> None:
    """c[:M, :N] (+)= A B^T over Z_{2^32} with B (N x K) given as ring words
    (an int32 tensor); A has at most 64 rows."""
    _need_dig(a, M, K, "a", optional=False)
    _need(b, N, K, "b", _INT, optional=False)
    _need(c, M, N, "c", _INT, optional=False)
    _check(_lib.load().mosaic_masked_matmul_words(a.ptr, a.pitch, b.data_ptr(), b.stride(0), M, N, K, c.data_ptr(),
                                                  c.stride(0), 1 if accumulate else 0, _stream()),
           "mosaic_masked_matmul_words")


def mosaic_integrity_check(ct: Digits, a: Digits, v: Digits, yq: torch.Tensor, t: int, M: int, K: int, NR: int,
                           d: torch.Tensor, count: torch.Tensor) -> None:
    """d = c^T A'^T - V [Y' | Q]^T (t x M) and count[0] = its nonzero entries,
    with [Y' | Q] given as the ring words of yq's first NR columns."""
    st = (_b or _native()).integrity_check(ct, a, v, yq, t, M, K, NR, d, count)
    if st is not None:
        return _check(st, "mosaic_integrity_check")
    _need_dig(ct, t, K, "ct", optional=False)
    _need_dig(a, M, K, "a", optional=False)
    _need_dig(v, t, NR, "v", optional=False)
    _need(yq, M, NR, "yq", _INT, optional=False)
    _need(d, t, M, "d", _INT, optional=False)
    if count.dtype != torch.int64 or count.numel() < 1 or not count.is_cuda:
        raise ValueError("count must be an int64 device tensor")
    _check(_lib.load().mosaic_integrity_check(ct.ptr, ct.pitch, a.ptr, a.pitch, v.ptr, v.pitch, yq.data_ptr(),
                                              yq.stride(0), t, M, K, NR, d.data_ptr(), d.stride(0),
                                              count.data_ptr(), _stream()), "mosaic_integrity_check")


def mosaic_unmask(ym: torch.Tensor, kc: Optional[torch.Tensor], q: Optional[Digits], l: Optional[Digits],
                  M: int, N: int, R: int, y: Optional[torch.Tensor] = None,
                  s_rows: Optional[torch.Tensor] = None, s_cols: Optional[torch.Tensor] = None,
                  y_f32: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None) -> None:
    st = (_b or _native()).unmask(ym, kc, q, l, M, N, R, y, s_rows, s_cols, y_f32, bias)
    if st is not None:
        return _check(st, "mosaic_unmask")
    _need(ym, M, N, "ym", _INT, optional=False)
    _need(kc, M, N, "kc", _INT)
    if R > 0:
        _need_dig(q, M, R, "q", optional=False)
        _need_dig(l, N, R, "l", optional=False)
    _need(y, M, N, "y", _INT)
    _need(y_f32, M, N, "y_f32", (torch.float32,))
    if y_f32 is not None:
        _need(s_rows, 1, M, "s_rows", (torch.float32,), optional=False)
        _need(s_cols, 1, N, "s_cols", (torch.float32,), optional=False)
    _need(bias, 1, N, "bias", (torch.float32,))
    _check(_lib.load().mosaic_unmask(ym.data_ptr(), ym.stride(0), _ptr(kc), kc.stride(0) if kc is not None else 0,
                                     q.ptr if q else None, q.pitch if q else 0,
                                     l.ptr if l else None, l.pitch if l else 0, M, N, R,
                                     _ptr(y), y.stride(0) if y is not None else 0,
                                     _ptr(s_rows), _ptr(s_cols), _ptr(bias), _ptr(y_f32),
                                     y_f32.stride(0) if y_f32 is not None else 0, _stream()), "mosaic_unmask")


def mosaic_unmask_words(ym: torch.Tensor, kc: Optional[torch.Tensor], q: Optional[torch.Tensor],
                        l: Optional[Digits], M: int, N: int, R: int, y: Optional[torch.Tensor] = None,
                        s_rows: Optional[torch.Tensor] = None, s_cols: Optional[torch.Tensor] = None,
                        y_f32: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None) -> None:
    """mosaic_unmask with q (M x R) as ring words, e.g. the Q columns of the
    server's [Y' | Q]; at most 16 rows."""
    st = (_b or _native()).unmask_words(ym, kc, q, l, M, N, R, y, s_rows, s_cols, y_f32, bias)
    if st is not None:
        return _check(st, "mosaic_unmask_words")
    _need(ym, M, N, "ym", _INT, optional=False)
    _need(kc, M, N, "kc", _INT)
    if R > 0:
        _need(q, M, R, "q", _INT, optional=False)
        _need_dig(l, N, R, "l", optional=False)
    _need(y, M, N, "y", _INT)
    _need(y_f32, M, N, "y_f32", (torch.float32,))
    if y_f32 is not None:
        _need(s_rows, 1, M, "s_rows", (torch.float32,), optional=False)
        _need(s_cols, 1, N, "s_cols", (torch.float32,), optional=False)
    _need(bias, 1, N, "bias", (torch.float32,))
    _check(_lib.load().mosaic_unmask_words(ym.data_ptr(), ym.stride(0), _ptr(kc),
                                           kc.stride(0) if kc is not None else 0,
                                           _ptr(q), q.stride(0) if q is not None else 0,
                                           l.ptr if l else None, l.pitch if l else 0, M, N, R,
                                           _ptr(y), y.stride(0) if y is not None else 0,
                                           _ptr(s_rows), _ptr(s_cols), _ptr(bias), _ptr(y_f32),
                                           y_f32.stride(0) if y_f32 is not None else 0, _stream()),
           "mosaic_unmask_words")


def mosaic_rotate_quantize_mask(x: torch.Tensor, qmax: int, out_dig: Digits, block: Optional[int] = None,
                                signs: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None,
                                noise: Optional[_lib.MosaicRng] = None,
                                scale: Optional[torch.Tensor] = None) -> None:
    """Fused rotate + quantise + mask of Pi_Sec-Linear's input: digits of
    round(R x / s) + u + noise for every row of x, and the row scales."""
    st = (_b or _native()).rotate_quantize_mask(x, qmax, out_dig, block, signs, u, noise, scale)
    if st is not None:
        return _check(st, "mosaic_rotate_quantize_mask")
    rows, n = x.shape
    _need(x, rows, n, "x", (torch.float32,), optional=False)
    _need_dig(out_dig, rows, n, "out_dig", optional=False)
    _need(u, rows, n, "u", _INT)
    _need(scale, 1, rows, "scale", (torch.float32,))
    _need(signs, 1, n, "signs", (torch.int8,))
    _check(_lib.load().mosaic_rotate_quantize_mask(x.data_ptr(), x.stride(0), rows, n, n if block is None else block,
                                                   _ptr(signs), qmax, _ptr(u), u.stride(0) if u is not None else 0,
                                                   ctypes.byref(noise) if noise is not None else None,
                                                   out_dig.ptr, out_dig.pitch, _ptr(scale), _stream()),
           "mosaic_rotate_quantize_mask")


@dataclass
class SparseRows:
    """Compressed rows of a sparse ring matrix (rows x cols) on the device."""
    row_ptr: torch.Tensor      # int64, rows + 1
    col_idx: torch.Tensor      # int32, capacity >= nnz
    values: torch.Tensor       # int32 holding uint32 ring values
    rows: int
    cols: int


def mosaic_sparse_csr(r: _lib.MosaicRng, rows: int, cols: int, exact: bool = True, device="cuda") -> SparseRows:
    """Compressed rows of the SPARSE or WEIGHT stream matrix of ``r``. With
    ``exact`` the arrays are sized to the nonzero count (one device-to-host
    read for SPARSE; rows * t for WEIGHT); otherwise to the bound rows * cols
    (no synchronisation)."""
    row_ptr = torch.empty(rows + 1, dtype=torch.int64, device=device)
    _check(_lib.load().mosaic_sparse_csr_count(ctypes.byref(r), rows, cols, row_ptr.data_ptr(), _stream()),
           "mosaic_sparse_csr_count")
    if r.dist == DIST_WEIGHT:
        cap = rows * r.row_weight
    else:
        cap = int(row_ptr[rows].item()) if exact else rows * cols
    col_idx = torch.empty(max(cap, 1), dtype=torch.int32, device=device)
    values = torch.empty(max(cap, 1), dtype=torch.int32, device=device)
    _check(_lib.load().mosaic_sparse_csr_fill(ctypes.byref(r), rows, cols, row_ptr.data_ptr(), col_idx.data_ptr(),
                                              values.data_ptr(), _stream()), "mosaic_sparse_csr_fill")
    return SparseRows(row_ptr, col_idx, values, rows, cols)


def mosaic_sparse_gather_rows(p: SparseRows, d: torch.Tensor, ncols: int, c: torch.Tensor,
                              subtract: bool = False) -> None:
    """c[i, :ncols] +-= sum_j P[i, j] d[j, :ncols] (P: rows x r sparse)."""
    _need(d, p.cols, ncols, "d", _INT, optional=False)
    _need(c, p.rows, ncols, "c", _INT, optional=False)
    _check(_lib.load().mosaic_sparse_gather_rows(p.rows, p.row_ptr.data_ptr(), p.col_idx.data_ptr(),
                                                 p.values.data_ptr(), d.data_ptr(), d.stride(0), ncols,
                                                 c.data_ptr(), c.stride(0), 1 if subtract else 0, _stream()),
           "mosaic_sparse_gather_rows")


def mosaic_sparse_stream_gather_rows(r: _lib.MosaicRng, rows: int, rcols: int, d: torch.Tensor, ncols: int,
                                     c: torch.Tensor, subtract: bool = False) -> None:
    """c[i, :ncols] +-= sum_j P[i, j] d[j, :ncols], P the rows x rcols SPARSE
    stream matrix of ``r`` (drawn inside the call)."""
    st = (_b or _native()).stream_terms([(r, rcols, d)], rows, ncols, c, subtract)
    if st is not None:
        return _check(st, "mosaic_sparse_stream_gather_rows")
    _need(d, rcols, ncols, "d", _INT, optional=False)
    _need(c, rows, ncols, "c", _INT, optional=False)
    _check(_lib.load().mosaic_sparse_stream_gather_rows(ctypes.byref(r), rows, rcols, d.data_ptr(), d.stride(0), ncols,
                                                        c.data_ptr(), c.stride(0), 1 if subtract else 0, _stream()),
           "mosaic_sparse_stream_gather_rows")


def mosaic_sparse_gather_cols(p: SparseRows, d: torch.Tensor, M: int, c: torch.Tensor,
                              subtract: bool = False, y_f32: Optional[torch.Tensor] = None,
                              s_rows: Optional[torch.Tensor] = None, s_cols: Optional[torch.Tensor] = None,
                              bias: Optional[torch.Tensor] = None) -> None:
    """c[m, n] +-= sum_j d[m, j] P[n, j] for m < M, n < P.rows; with y_f32,
    also y_f32 = c s_rows[m] s_cols[n] (+ bias[n]) of the finished c."""
    N = p.rows
    _need(d, M, p.cols, "d", _INT, optional=False)
    _need(c, M, N, "c", _INT, optional=False)
    _need(y_f32, M, N, "y_f32", (torch.float32,))
    if y_f32 is not None:
        _need(s_rows, 1, M, "s_rows", (torch.float32,), optional=False)
        _need(s_cols, 1, N, "s_cols", (torch.float32,), optional=False)
    _need(bias, 1, N, "bias", (torch.float32,))
    _check(_lib.load().mosaic_sparse_gather_cols(M, N, p.row_ptr.data_ptr(), p.col_idx.data_ptr(),
                                                 p.values.data_ptr(), d.data_ptr(), d.stride(0), c.data_ptr(),
                                                 c.stride(0), 1 if subtract else 0, _ptr(s_rows), _ptr(s_cols),
                                                 _ptr(bias), _ptr(y_f32), y_f32.stride(0) if y_f32 is not None else 0,
                                                 _stream()),
           "mosaic_sparse_gather_cols")


def mosaic_sparse_stream_gather_rows_terms(terms: Sequence[Tuple[_lib.MosaicRng, int, torch.Tensor]], rows: int,
                                           ncols: int, c: torch.Tensor, subtract: bool = False) -> None:
    """c[i, :ncols] +-= the sum over the terms (r, rcols, d) of
    mosaic_sparse_stream_gather_rows, in one call."""
    st = (_b or _native()).stream_terms(terms, rows, ncols, c, subtract)
    if st is not None:
        return _check(st, "mosaic_sparse_stream_gather_rows_terms")
    _need(c, rows, ncols, "c", _INT, optional=False)
    arr = (_lib.MosaicStreamTerm * max(1, len(terms)))()
    for t, (r, rcols, d) in zip(arr, terms):
        _need(d, rcols, ncols, "d", _INT, optional=False)
        t.rng, t.rcols, t.d, t.ldd = r, rcols, d.data_ptr(), d.stride(0)
    _check(_lib.load().mosaic_sparse_stream_gather_rows_terms(arr, len(terms), rows, ncols, c.data_ptr(), c.stride(0),
                                                              1 if subtract else 0, _stream()),
           "mosaic_sparse_stream_gather_rows_terms")


def mosaic_sparse_gather_cols_terms(terms: Sequence[Tuple[SparseRows, torch.Tensor]], M: int, c: torch.Tensor,
                                    subtract: bool = False, y_f32: Optional[torch.Tensor] = None,
                                    s_rows: Optional[torch.Tensor] = None, s_cols: Optional[torch.Tensor] = None,
                                    bias: Optional[torch.Tensor] = None) -> None:
    """c[m, n] +-= the sum over the terms (p, d) of mosaic_sparse_gather_cols,
    in one call; y_f32 as there."""
    st = (_b or _native()).cols_terms(terms, M, c, subtract, y_f32, s_rows, s_cols, bias)
    if st is not None:
        return _check(st, "mosaic_sparse_gather_cols_terms")
    N = terms[0][0].rows
    _need(c, M, N, "c", _INT, optional=False)
    _need(y_f32, M, N, "y_f32", (torch.float32,))
    if y_f32 is not None:
        _need(s_rows, 1, M, "s_rows", (torch.float32,), optional=False)
        _need(s_cols, 1, N, "s_cols", (torch.float32,), optional=False)
    _need(bias, 1, N, "bias", (torch.float32,))
    arr = (_lib.MosaicSparseTerm * len(terms))()
    for t, (p, d) in zip(arr, terms):
        if p.rows != N:
            raise ValueError("the terms' matrices have different row counts")
        _need(d, M, p.cols, "d", _INT, optional=False)
        t.row_ptr, t.col_idx, t.values = p.row_ptr.data_ptr(), p.col_idx.data_ptr(), p.values.data_ptr()
        t.cols, t.d, t.ldd = p.cols, d.data_ptr(), d.stride(0)
    _check(_lib.load().mosaic_sparse_gather_cols_terms(arr, len(terms), M, N, c.data_ptr(), c.stride(0),
                                                       1 if subtract else 0, _ptr(s_rows), _ptr(s_cols), _ptr(bias),
                                                       _ptr(y_f32), y_f32.stride(0) if y_f32 is not None else 0,
                                                       _stream()), "mosaic_sparse_gather_cols_terms")


def mosaic_count_mismatches(a: torch.Tensor, b: torch.Tensor, count: torch.Tensor) -> None:
    """count[0] = number of entries where the int32 matrices a and b differ
    (same shape; count is a one-element int64 device tensor)."""
    if a.shape != b.shape or a.dim() != 2:
        raise ValueError("a and b must be matrices of the same shape")
    if count.dtype != torch.int64 or count.numel() < 1:
        raise ValueError("count must be an int64 tensor")
    rows, cols = a.shape
    _check(_lib.load().mosaic_count_mismatches(a.data_ptr(), a.stride(0), b.data_ptr(), b.stride(0), rows, cols,
                                               count.data_ptr(), _stream()), "mosaic_count_mismatches")


def mosaic_sample_signs(r: _lib.MosaicRng, n: int, out: torch.Tensor) -> None:
    _need(out, 1, n, "out", (torch.int8,), optional=False)
    _check(_lib.load().mosaic_sample_signs(ctypes.byref(r), n, out.data_ptr(), _stream()), "mosaic_sample_signs")


def mosaic_hadamard_rotate(x: torch.Tensor, y: torch.Tensor, block: Optional[int] = None,
                           signs: Optional[torch.Tensor] = None, inverse: bool = False) -> None:
    st = (_b or _native()).hadamard_rotate(x, y, block, signs, inverse)
    if st is not None:
        return _check(st, "mosaic_hadamard_rotate")
    rows, n = x.shape
    _need(x, rows, n, "x", (torch.float32,), optional=False)
    _need(y, rows, n, "y", (torch.float32,), optional=False)
    _need(signs, 1, n, "signs", (torch.int8,))
    _check(_lib.load().mosaic_hadamard_rotate(x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), rows, n,
                                              n if block is None else block, _ptr(signs), 1 if inverse else 0,
                                              _stream()), "mosaic_hadamard_rotate")


def mosaic_hadamard28_rotate(x: torch.Tensor, y: torch.Tensor, signs: Optional[torch.Tensor] = None,
                             inverse: bool = False) -> None:
    rows, n = x.shape
    _need(x, rows, n, "x", (torch.float32,), optional=False)
    _need(y, rows, n, "y", (torch.float32,), optional=False)
    _need(signs, 1, n, "signs", (torch.int8,))
    _check(_lib.load().mosaic_hadamard28_rotate(x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), rows, n,
                                                _ptr(signs), 1 if inverse else 0, _stream()),
           "mosaic_hadamard28_rotate")


def mosaic_quantize_rows(x: torch.Tensor, qmax: int, q: Optional[torch.Tensor] = None,
                         q_dig: Optional[Digits] = None, scale: Optional[torch.Tensor] = None) -> None:
    st = (_b or _native()).quantize_rows(x, qmax, q, q_dig, scale)
    if st is not None:
        return _check(st, "mosaic_quantize_rows")
    rows, n = x.shape
    _need(x, rows, n, "x", (torch.float32,), optional=False)
    _need(q, rows, n, "q", _INT)
    _need_dig(q_dig, rows, n, "q_dig")
    _need(scale, 1, rows, "scale", (torch.float32,))
    _check(_lib.load().mosaic_quantize_rows(x.data_ptr(), x.stride(0), rows, n, qmax, _ptr(q),
                                            q.stride(0) if q is not None else 0,
                                            q_dig.ptr if q_dig else None, q_dig.pitch if q_dig else 0,
                                            _ptr(scale), _stream()), "mosaic_quantize_rows")


@dataclass
class KVCache:
    """Keys and values of a batch of sequences in pages (include/mosaic_cache.h).

    ``k`` and ``v`` have shape (pages, kv_heads, page_size, head_dim) and the
    same strides, with contiguous rows: a view of memory that is laid out
    (pages, page_size, kv_heads, head_dim) will do. ``block_table`` (int32,
    batch x blocks) holds every sequence's pages, ``state`` (int32, 2 x batch)
    how many tokens it holds and how many it has seen. ``weights`` (float32)
    and ``order`` (int32), contiguous (pages, kv_heads, page_size), are needed
    for eviction only."""
    k: torch.Tensor
    v: torch.Tensor
    block_table: torch.Tensor
    state: torch.Tensor
    weights: Optional[torch.Tensor] = None
    order: Optional[torch.Tensor] = None

    @staticmethod
    def empty(batch: int, max_len: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, page_size: int = 64,
              evicts: bool = False, device="cuda") -> "KVCache":
        """A cache without tokens, with pages of its own for ``max_len`` slots
        of each sequence."""
        blocks = (max_len + page_size - 1) // page_size
        pages = batch * blocks
        k = torch.empty((pages, kv_heads, page_size, head_dim), dtype=dtype, device=device)
        table = torch.arange(pages, dtype=torch.int32, device=device).reshape(batch, blocks)
        state = torch.zeros((2, batch), dtype=torch.int32, device=device)
        weights = torch.zeros(k.shape[:3], device=device) if evicts else None
        order = torch.zeros(k.shape[:3], dtype=torch.int32, device=device) if evicts else None
        return KVCache(k, torch.empty_like(k), table, state, weights, order)

    @property
    def batch(self) -> int:
        return self.block_table.shape[0]

    @property
    def slots(self) -> int:
        """Tokens that a sequence's block table has room for."""
        return self.block_table.shape[1] * self.k.shape[2]


@dataclass
class Rotary:
    """Rotary positions: ``table`` (float32, rows x 2P) holds cosines and sines
    by place and pair, ``sections`` the pairs of each axis (their sum is P),
    ``positions`` (int32, axes x tokens) each new token's places; None: its
    number in its sequence. Pairs are the elements j and P + j of a head, or
    2j and 2j + 1 if ``interleaved``."""
    table: torch.Tensor
    sections: Sequence[int]
    positions: Optional[torch.Tensor] = None
    interleaved: bool = False

    @staticmethod
    def frequencies(rows: int, pairs: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
        """The table of angles place * base^(-j / pairs), from float64."""
        f = base ** (-torch.arange(pairs, dtype=torch.float64, device=device) / pairs)
        a = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * f
        return torch.cat([a.cos(), a.sin()], dim=1).float()


_FTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _device_tensor(t, name: str, dtypes, dim: int) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has dtype {t.dtype}, expected one of {tuple(dtypes)}")
    if t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions")


def _cache_arg(cache: KVCache) -> _lib.MosaicKvCache:
    """The C struct of a cache whose tensors fit together."""
    k, v, table = cache.k, cache.v, cache.block_table
    _device_tensor(k, "cache.k", _FTYPE, 4)
    _device_tensor(v, "cache.v", _FTYPE, 4)
    if v.dtype != k.dtype or v.shape != k.shape or v.stride() != k.stride():
        raise ValueError("cache.k and cache.v must have the same type, shape and strides")
    if k.stride(3) != 1:
        raise ValueError("rows of cache.k and cache.v must be contiguous")
    _device_tensor(table, "cache.block_table", _INT, 2)
    if table.shape[1] > 1 and table.stride(1) != 1:
        raise ValueError("rows of cache.block_table must be contiguous")
    batch, blocks = table.shape
    _device_tensor(cache.state, "cache.state", _INT, 2)
    if tuple(cache.state.shape) != (2, batch) or not cache.state.is_contiguous():
        raise ValueError("cache.state must be a contiguous (2, batch) tensor")
    for name, t, dt in (("weights", cache.weights, torch.float32), ("order", cache.order, torch.int32)):
        if t is not None:
            _device_tensor(t, f"cache.{name}", (dt,), 3)
            if t.shape != k.shape[:3] or not t.is_contiguous():
                raise ValueError(f"cache.{name} must be a contiguous (pages, kv_heads, page_size) tensor")
    pages, heads, page, dim = k.shape
    # a single row's stride has no meaning; 0 is a table that all sequences share
    return _lib.MosaicKvCache(k=_ptr(k), v=_ptr(v), weights=_ptr(cache.weights), order=_ptr(cache.order),
                              block_table=_ptr(table), ldt=table.stride(0) if batch > 1 else blocks, pages=pages,
                              page_stride=k.stride(0), head_stride=k.stride(1), token_stride=k.stride(2),
                              dtype=_FTYPE[k.dtype], batch=batch, max_blocks=blocks, kv_heads=heads, head_dim=dim,
                              page_size=page)


def _cache_rows(t: torch.Tensor, rows: int, cols: int, name: str, cache: KVCache) -> None:
    _device_tensor(t, name, (torch.float32, cache.k.dtype), 2)
    if t.shape[0] < rows or t.shape[1] < cols:
        raise ValueError(f"{name} is {tuple(t.shape)}, needs at least ({rows}, {cols})")
    if t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")


def _same_shape(t: Optional[torch.Tensor], like: Optional[torch.Tensor], name: str) -> Optional[torch.Tensor]:
    if t is None:
        return like
    if like is None:
        raise ValueError(f"{name} has no counterpart in the cache")
    _device_tensor(t, name, (like.dtype,), like.dim())
    if t.shape != like.shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {tuple(like.shape)} tensor")
    return t


def mosaic_cache_append(cache: KVCache, qkv: torch.Tensor, heads: int, q_out: torch.Tensor,
                        starts: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None,
                        new_state: Optional[torch.Tensor] = None) -> None:
    """New tokens, one per row of qkv (queries, keys, values of ``heads`` and
    kv_heads heads): rotated queries to q_out, rotated keys and values into
    the cache. Rows starts[b] .. starts[b + 1] - 1 are sequence b's (None: row
    b). The state is advanced in place unless new_state is given."""
    st = (_b or _native()).cache_append(cache, qkv, heads, q_out, starts, rotary, new_state)
    if st is not None:
        return _check(st, "mosaic_cache_append")
    c = _cache_arg(cache)
    rows = qkv.shape[0]
    _cache_rows(qkv, rows, (heads + 2 * c.kv_heads) * c.head_dim, "qkv", cache)
    _cache_rows(q_out, rows, heads * c.head_dim, "q_out", cache)
    if q_out.dtype != qkv.dtype:
        raise ValueError("q_out must have the type of qkv")
    if starts is not None:
        _device_tensor(starts, "starts", _INT, 1)
        if starts.shape[0] != c.batch + 1 or starts.stride(0) != 1:
            raise ValueError("starts must be a contiguous vector of batch + 1 entries")
    state = _same_shape(new_state, cache.state, "new_state")
    r = None
    if rotary is not None:
        sections = [int(n) for n in rotary.sections]
        if not 1 <= len(sections) <= 4:
            raise ValueError("rotary positions have one to four axes")
        _device_tensor(rotary.table, "rotary.table", (torch.float32,), 2)
        if rotary.table.shape[1] != 2 * sum(sections) or not rotary.table.is_contiguous():
            raise ValueError("rotary.table must be contiguous, with a cosine and a sine for every pair")
        if rotary.positions is not None:
            _device_tensor(rotary.positions, "rotary.positions", _INT, 2)
            if rotary.positions.shape[0] < len(sections) or rotary.positions.shape[1] < rows or \
                    (rows > 1 and rotary.positions.stride(1) != 1):
                raise ValueError("rotary.positions must hold a row of places for every axis")
        # 0: places that all axes share
        ldp = 0 if rotary.positions is None else rotary.positions.stride(0) if len(sections) > 1 else rows
        r = _lib.MosaicRotary(table=_ptr(rotary.table), rows=rotary.table.shape[0], positions=_ptr(rotary.positions), ldp=ldp,
                              naxes=len(sections), sections=(ctypes.c_int32 * 4)(*sections),
                              interleaved=1 if rotary.interleaved else 0)
    _check(_lib.load().mosaic_cache_append(ctypes.byref(c), _ptr(qkv), qkv.stride(0), _FTYPE[qkv.dtype], rows,
                                           _ptr(starts), heads, None if r is None else ctypes.byref(r), _ptr(q_out),
                                           q_out.stride(0), _ptr(cache.state), _ptr(state), _stream()),
           "mosaic_cache_append")


def mosaic_cache_attend(cache: KVCache, q: torch.Tensor, heads: int, out: torch.Tensor,
                        max_len: Optional[int] = None, scale: Optional[float] = None,
                        accumulate: bool = False) -> None:
    """out[b] = attention of q[b] (one new token, ``heads`` heads) over the
    tokens that sequence b holds; ``accumulate`` adds the attention weights
    up in cache.weights. ``max_len``: no sequence holds more tokens (None: as
    many as there are slots); with ``accumulate`` the call takes batch x heads
    x max_len floats of memory for its scores. ``scale`` defaults to 1 /
    sqrt(head_dim)."""
    st = (_b or _native()).cache_attend(cache, q, heads, out, max_len, scale, accumulate)
    if st is not None:
        return _check(st, "mosaic_cache_attend")
    c = _cache_arg(cache)
    _cache_rows(q, c.batch, heads * c.head_dim, "q", cache)
    _cache_rows(out, c.batch, heads * c.head_dim, "out", cache)
    if out.dtype != q.dtype:
        raise ValueError("out must have the type of q")
    if accumulate and cache.weights is None:
        raise ValueError("the cache has no weights to add to")
    n = cache.slots if max_len is None else max_len
    lib, size = _lib.load(), ctypes.c_int64(0)
    _check(lib.mosaic_cache_attend_workspace(ctypes.byref(c), heads, n, 1 if accumulate else 0, ctypes.byref(size)),
           "mosaic_cache_attend_workspace")
    work = torch.empty(size.value, dtype=torch.uint8, device=q.device)
    _check(lib.mosaic_cache_attend(ctypes.byref(c), _ptr(q), q.stride(0), _FTYPE[q.dtype], heads, _ptr(cache.state), n,
                                   c.head_dim ** -0.5 if scale is None else scale, 1 if accumulate else 0, _ptr(out),
                                   out.stride(0), _ptr(work), size.value, _stream()), "mosaic_cache_attend")


def mosaic_cache_evict(cache: KVCache, budget: int, recent: int, max_len: Optional[int] = None,
                       new_state: Optional[torch.Tensor] = None, new_weights: Optional[torch.Tensor] = None,
                       new_order: Optional[torch.Tensor] = None, kept: Optional[torch.Tensor] = None) -> None:
    """Every sequence that holds more than ``budget`` tokens keeps, for each
    key/value head, the ``recent`` latest and the ones with the largest
    weights, moved into its first ``budget`` slots. Weights, order and state
    change in place unless others are given; ``kept`` (int32, batch x kv_heads
    x budget) gets the slot that each slot's token had before."""
    st = (_b or _native()).cache_evict(cache, budget, recent, max_len, new_state, new_weights, new_order, kept)
    if st is not None:
        return _check(st, "mosaic_cache_evict")
    c = _cache_arg(cache)
    if cache.weights is None or cache.order is None:
        raise ValueError("eviction needs a cache with weights and order")
    state = _same_shape(new_state, cache.state, "new_state")
    weights = _same_shape(new_weights, cache.weights, "new_weights")
    order = _same_shape(new_order, cache.order, "new_order")
    if kept is not None:
        _device_tensor(kept, "kept", _INT, 3)
        if tuple(kept.shape) != (c.batch, c.kv_heads, budget) or not kept.is_contiguous():
            raise ValueError("kept must be a contiguous (batch, kv_heads, budget) tensor")
    n = cache.slots if max_len is None else max_len
    lib, size = _lib.load(), ctypes.c_int64(0)
    _check(lib.mosaic_cache_evict_workspace(ctypes.byref(c), n, budget, ctypes.byref(size)),
           "mosaic_cache_evict_workspace")
    work = torch.empty(size.value, dtype=torch.uint8, device=cache.k.device)
    _check(lib.mosaic_cache_evict(ctypes.byref(c), _ptr(cache.state), _ptr(state), n, budget, recent, _ptr(weights),
                                  _ptr(order), _ptr(kept), _ptr(work), size.value, _stream()), "mosaic_cache_evict")


def mosaic_probe_mfma_i8(mode: int, iters: int, out: torch.Tensor) -> int:
    """Launches the register-only MFMA probe (measurement aid); returns the
    int8 operations launched. ``out`` is a one-element int32 device tensor."""
    ops = ctypes.c_int64(0)
    _check(_lib.load().mosaic_probe_mfma_i8(mode, iters, out.data_ptr(), ctypes.byref(ops), _stream()),
           "mosaic_probe_mfma_i8")
    return int(ops.value)
