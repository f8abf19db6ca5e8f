"""Torch-tensor front end of the C ABI (same names as include/maddness.h).

Each function checks dtypes, devices and shapes, allocates outputs that were
not supplied, and passes raw device pointers plus the current HIP stream to
the library.  No arithmetic of the method happens here.

With ``validate=True`` the device-array preconditions of the ABI (split
columns in range, indices below 16, scales exact powers of two, no int32
overflow) are checked on host copies first; this synchronises and is meant
for tests and debugging.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import NamedTuple, Optional, Tuple

import torch

from . import _lib

K, LEVELS, NODES = 16, 4, 15


def _ptr(t: Optional[torch.Tensor]):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _stream(stream) -> ctypes.c_void_p:
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, ndim: int):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _dense(t: torch.Tensor, name: str):
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _rows(A: torch.Tensor) -> Tuple[int, int, int]:
    _need(A, "A", torch.float32, 2)
    if A.shape[0] > 1 and A.stride(1) != 1:
        raise ValueError("A must have unit column stride")
    N, D = A.shape
    lda = A.stride(0) if N > 1 else D
    return N, D, lda


def _native(A, split, thr, lut, scale, offset, col_bias, act, y_out, acc_out, idx_out, want_acc, want_idx):
    """The call marshalled natively, on the current stream: (y, acc, idx), or
    None when the arguments are not the plain valid case (the caller then goes
    through its own checks, which raise), the call reports an error or there
    is no native marshalling."""
    if type(A) is not torch.Tensor or not A.is_cuda or not (act is None or type(act) is int):
        return None
    fused = _fused if _fused is not None else _load_native()
    if not fused:
        return None
    return fused(A, split, thr, lut, scale, offset, col_bias, act, y_out, acc_out, idx_out, want_acc, want_idx,
                 torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()))


_fused = None


def _load_native():
    global _fused
    calls = _lib.calls()
    _fused = calls.fused if calls else False
    return _fused


def _tree_args(split: torch.Tensor, thr: torch.Tensor) -> int:
    _need(split, "split_dims", torch.int32, 2)
    _need(thr, "thresholds", torch.float32, 2)
    _dense(split, "split_dims")
    _dense(thr, "thresholds")
    C = split.shape[0]
    if tuple(split.shape) != (C, LEVELS) or tuple(thr.shape) != (C, NODES):
        raise ValueError(f"split_dims must be [C,4] and thresholds [C,15], got "
                         f"{tuple(split.shape)} and {tuple(thr.shape)}")
    return C


def _validate_trees(split: torch.Tensor, D: int):
    s = split.cpu()
    if s.numel() and (int(s.min()) < 0 or int(s.max()) >= D):
        raise ValueError("split_dims outside [0, D)")


def _validate_scales(scale: torch.Tensor):
    s = scale.cpu().numpy()
    import numpy as np
    m, e = np.frexp(s)
    if not (np.all(m == 0.5) and np.all(e - 1 >= -126)):
        raise ValueError("scales must be exact normal powers of two")
    sh = (e - 1) - (e - 1).min()
    if np.any(sh > 30) or float(np.sum(128.0 * np.ldexp(1.0, sh))) > 2.0 ** 31:
        raise ValueError("scale exponents too far apart: a sum of int8 codes could leave int32")


def _validate_idx(idx: torch.Tensor):
    if idx.numel() and int(idx.max()) >= K:
        raise ValueError("indices must lie in [0, 16)")


def encode(A, split_dims, thresholds, idx_out=None, stream=None, validate=False):
    """Tree encoding: returns idx [N][C] uint8 (see maddness_encode)."""
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    if validate:
        _validate_trees(split_dims, D)
    if idx_out is None:
        idx_out = torch.empty((N, C), dtype=torch.uint8, device=A.device)
    _need(idx_out, "idx_out", torch.uint8, 2)
    _dense(idx_out, "idx_out")
    st = _lib.lib().maddness_encode(_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C,
                                    _ptr(idx_out), _stream(stream))
    _lib.check("maddness_encode", st)
    return idx_out


def _lut_i8(lut, scale, offset):
    _need(lut, "lut", torch.int8, 3)
    _need(scale, "scale", torch.float32, 1)
    _need(offset, "offset", torch.float32, 1)
    for t, n in ((lut, "lut"), (scale, "scale"), (offset, "offset")):
        _dense(t, n)
    C, k, M = lut.shape
    if k != K or scale.shape[0] != C or offset.shape[0] != C:
        raise ValueError("lut must be [C,16,M], scale and offset [C]")
    return C, M


def lut_accumulate(idx, lut, scale, offset, acc_out=None, y_out=None, want_acc=False, want_y=True,
                   stream=None, validate=False):
    """Gather-accumulate over an int8 block-FP table; returns (acc or None, y or None)."""
    _need(idx, "idx", torch.uint8, 2)
    _dense(idx, "idx")
    C, M = _lut_i8(lut, scale, offset)
    N = idx.shape[0]
    if idx.shape[1] != C:
        raise ValueError("idx must be [N, C]")
    if validate:
        _validate_idx(idx)
        _validate_scales(scale)
    if acc_out is None and want_acc:
        acc_out = torch.empty((N, M), dtype=torch.int32, device=idx.device)
    if y_out is None and want_y:
        y_out = torch.empty((N, M), dtype=torch.float32, device=idx.device)
    st = _lib.lib().maddness_lut_accumulate(_ptr(idx), N, C, _ptr(lut), _ptr(scale), _ptr(offset), M,
                                            _ptr(acc_out), _ptr(y_out), _stream(stream))
    _lib.check("maddness_lut_accumulate", st)
    return acc_out, y_out


def lut_accumulate_avg(idx, lut, scale, offset, acc_out=None, y_out=None, want_acc=False, want_y=True,
                       stream=None, validate=False):
    """Rounded 8-bit summation over codebooks (approximate; one shared scale);
    returns (acc or None, y or None)."""
    _need(idx, "idx", torch.uint8, 2)
    _dense(idx, "idx")
    C, M = _lut_i8(lut, scale, offset)
    N = idx.shape[0]
    if idx.shape[1] != C:
        raise ValueError("idx must be [N, C]")
    if validate:
        _validate_idx(idx)
        _validate_scales(scale)
        if not bool((scale == scale[0]).all()):
            raise ValueError("the averaging accumulate needs one scale shared by every codebook")
    if acc_out is None and want_acc:
        acc_out = torch.empty((N, M), dtype=torch.int32, device=idx.device)
    if y_out is None and want_y:
        y_out = torch.empty((N, M), dtype=torch.float32, device=idx.device)
    st = _lib.lib().maddness_lut_accumulate_avg(_ptr(idx), N, C, _ptr(lut), _ptr(scale), _ptr(offset), M,
                                                _ptr(acc_out), _ptr(y_out), _stream(stream))
    _lib.check("maddness_lut_accumulate_avg", st)
    return acc_out, y_out


def lut_accumulate_f32(idx, lut, y_out=None, stream=None, validate=False):
    """Gather-accumulate over an fp32 table [C][16][M]; returns y [N][M]."""
    _need(idx, "idx", torch.uint8, 2)
    _need(lut, "lut", torch.float32, 3)
    _dense(idx, "idx")
    _dense(lut, "lut")
    C, k, M = lut.shape
    N = idx.shape[0]
    if k != K or idx.shape[1] != C:
        raise ValueError("lut must be [C,16,M] and idx [N,C]")
    if validate:
        _validate_idx(idx)
    if y_out is None:
        y_out = torch.empty((N, M), dtype=torch.float32, device=idx.device)
    st = _lib.lib().maddness_lut_accumulate_f32(_ptr(idx), N, C, _ptr(lut), M, _ptr(y_out),
                                                _stream(stream))
    _lib.check("maddness_lut_accumulate_f32", st)
    return y_out


def matmul(A, split_dims, thresholds, lut, scale, offset, y_out=None, acc_out=None, idx_out=None,
           want_acc=False, want_idx=False, stream=None, validate=False):
    """Fused encode + int8 lookup-accumulate; returns (y, acc or None, idx or None)."""
    if stream is None and validate is False and scale is not None:
        r = _native(A, split_dims, thresholds, lut, scale, offset, None, None, y_out, acc_out, idx_out, want_acc, want_idx)
        if r is not None:
            return r
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    C2, M = _lut_i8(lut, scale, offset)
    if C2 != C:
        raise ValueError("lut codebooks differ from the trees'")
    if validate:
        _validate_trees(split_dims, D)
        _validate_scales(scale)
    dev = A.device
    if y_out is None:
        y_out = torch.empty((N, M), dtype=torch.float32, device=dev)
    if acc_out is None and want_acc:
        acc_out = torch.empty((N, M), dtype=torch.int32, device=dev)
    if idx_out is None and want_idx:
        idx_out = torch.empty((N, C), dtype=torch.uint8, device=dev)
    idx_out = _idx_out(idx_out, N, C)
    idx_arg = _index_array(idx_out, A, N, D, lda, C, M, False, 0, stream)
    st = _lib.lib().maddness_matmul(_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C,
                                    _ptr(lut), _ptr(scale), _ptr(offset), M, _ptr(y_out),
                                    _ptr(acc_out), _ptr(idx_arg), _stream(stream))
    _lib.check("maddness_matmul", st)
    return y_out, acc_out, idx_out


def matmul_noalloc(A, split_dims, thresholds, lut, scale, offset, y_out, acc_out=None, idx_out=None,
                   stream=None):
    """maddness_matmul_noalloc: the fused int8 path with every buffer given
    by the caller (y_out required) and, for large tables without idx_out,
    the library's static scratch array in place of an index array; neither
    this function nor the library allocates.  Returns y_out."""
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    C2, M = _lut_i8(lut, scale, offset)
    if C2 != C:
        raise ValueError("lut codebooks differ from the trees'")
    _need(y_out, "y_out", torch.float32, 2)
    _dense(y_out, "y_out")
    if tuple(y_out.shape) != (N, M):
        raise ValueError("y_out must be [N, M]")
    if acc_out is not None:
        _need(acc_out, "acc_out", torch.int32, 2)
        _dense(acc_out, "acc_out")
        if tuple(acc_out.shape) != (N, M):
            raise ValueError("acc_out must be [N, M]")
    idx_out = _idx_out(idx_out, N, C)
    st = _lib.lib().maddness_matmul_noalloc(_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C,
                                            _ptr(lut), _ptr(scale), _ptr(offset), M, _ptr(y_out),
                                            _ptr(acc_out), _ptr(idx_out), _stream(stream))
    _lib.check("maddness_matmul_noalloc", st)
    return y_out


def matmul_f32(A, split_dims, thresholds, lut, y_out=None, idx_out=None, want_idx=False, stream=None,
               validate=False):
    """Fused encode + fp32 lookup-accumulate; returns (y, idx or None)."""
    if stream is None and validate is False:
        r = _native(A, split_dims, thresholds, lut, None, None, None, None, y_out, None, idx_out, False, want_idx)
        if r is not None:
            return r[0], r[2]
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    _need(lut, "lut", torch.float32, 3)
    _dense(lut, "lut")
    if lut.shape[0] != C or lut.shape[1] != K:
        raise ValueError("lut must be [C,16,M]")
    M = lut.shape[2]
    if validate:
        _validate_trees(split_dims, D)
    if y_out is None:
        y_out = torch.empty((N, M), dtype=torch.float32, device=A.device)
    if idx_out is None and want_idx:
        idx_out = torch.empty((N, C), dtype=torch.uint8, device=A.device)
    idx_out = _idx_out(idx_out, N, C)
    idx_arg = _index_array(idx_out, A, N, D, lda, C, M, True, 0, stream)
    st = _lib.lib().maddness_matmul_f32(_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C,
                                        _ptr(lut), M, _ptr(y_out), _ptr(idx_arg), _stream(stream))
    _lib.check("maddness_matmul_f32", st)
    return y_out, idx_out


ACT = {"none": 0, "bias": 1, "relu": 2, "softmax": 3}
# objectives of fit_lut_gd (MADDNESS_FIT_*): the layer output and the loss
FIT = {"relu": 2, "softmax": 3, "softmax_kld": 3, "softmax_sqerr": 4}


def _act(act):
    if isinstance(act, str):
        if act not in ACT:
            raise ValueError(f"act must be one of {sorted(ACT)}")
        return ACT[act]
    return int(act)


def _act_code(act):
    """act as an int, or something _native declines (never None)."""
    return ACT.get(act, "") if isinstance(act, str) else "" if act is None else act


def _col_bias(col_bias, M):
    if col_bias is None:
        return None
    _need(col_bias, "col_bias", torch.float32, 1)
    _dense(col_bias, "col_bias")
    if col_bias.shape[0] != M:
        raise ValueError("col_bias must be [M]")
    return col_bias


def _idx_out(idx_out, N, C):
    if idx_out is not None:
        _need(idx_out, "idx_out", torch.uint8, 2)
        _dense(idx_out, "idx_out")
        if tuple(idx_out.shape) != (N, C):
            raise ValueError("idx_out must be [N, C]")
    return idx_out


def matmul_index_bytes(A, C, M, f32=False, act=0) -> int:
    """Device bytes of idx_out the fused entry points use for this A and
    shape (maddness_matmul_index_bytes): 0 when the call runs as one launch,
    else N * C (the two-phase path; for the shapes that also have a slower
    one-launch route, the faster one through the index array)."""
    N, D, lda = _rows(A)
    n = int(_lib.lib().maddness_matmul_index_bytes(_ptr(A), N, D, lda, C, M, 1 if f32 else 0, _act(act)))
    if n < 0:
        _lib.check("maddness_matmul_index_bytes", _lib.EINVAL if n == -1 else _lib.EUNSUPPORTED)
    return n


def _index_array(idx_out, A, N, D, lda, C, M, f32, act, stream):
    """idx_out when the caller gave one; else, when the call uses an index
    array (the table does not fit the single-launch kernels, or two phases
    through it are faster), a new one from torch's allocator, kept alive for
    `stream`; else None.  The library itself never allocates."""
    if idx_out is not None:
        return idx_out
    n = int(_lib.lib().maddness_matmul_index_bytes(_ptr(A), N, D, lda, C, M, 1 if f32 else 0, int(act)))
    if n <= 0:
        return None   # one launch, or arguments the call itself rejects
    t = torch.empty((N, C), dtype=torch.uint8, device=A.device)
    if stream is not None:
        t.record_stream(stream)
    return t


def matmul_act(A, split_dims, thresholds, lut, scale, offset, col_bias=None, act="relu", y_out=None,
               idx_out=None, stream=None, validate=False):
    """Fused encode + lookup-accumulate + layer output sigma (bias, then
    "relu" / "softmax"; "bias" or "none" also accepted); returns y.  With
    idx_out the indices are written there; without it an index array is
    allocated here when the shape needs one (matmul_index_bytes)."""
    if stream is None and validate is False and scale is not None:
        r = _native(A, split_dims, thresholds, lut, scale, offset, col_bias, _act_code(act), y_out, None, idx_out,
                    False, False)
        if r is not None:
            return r[0]
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    C2, M = _lut_i8(lut, scale, offset)
    if C2 != C:
        raise ValueError("lut codebooks differ from the trees'")
    col_bias = _col_bias(col_bias, M)
    if validate:
        _validate_trees(split_dims, D)
        _validate_scales(scale)
    if y_out is None:
        y_out = torch.empty((N, M), dtype=torch.float32, device=A.device)
    _need(y_out, "y_out", torch.float32, 2)
    _dense(y_out, "y_out")
    idx_out = _idx_out(idx_out, N, C)
    idx_arg = _index_array(idx_out, A, N, D, lda, C, M, False, _act(act), stream)
    st = _lib.lib().maddness_matmul_act(_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C, _ptr(lut),
                                        _ptr(scale), _ptr(offset), M, _ptr(col_bias), _act(act), _ptr(y_out),
                                        _ptr(idx_arg), _stream(stream))
    _lib.check("maddness_matmul_act", st)
    return y_out


def matmul_act_f32(A, split_dims, thresholds, lut, col_bias=None, act="relu", y_out=None, idx_out=None,
                   stream=None, validate=False):
    """matmul_act over an unquantized fp32 table; returns y."""
    if stream is None and validate is False:
        r = _native(A, split_dims, thresholds, lut, None, None, col_bias, _act_code(act), y_out, None, idx_out,
                    False, False)
        if r is not None:
            return r[0]
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    _need(lut, "lut", torch.float32, 3)
    _dense(lut, "lut")
    if lut.shape[0] != C or lut.shape[1] != K:
        raise ValueError("lut must be [C,16,M]")
    M = lut.shape[2]
    col_bias = _col_bias(col_bias, M)
    if validate:
        _validate_trees(split_dims, D)
    if y_out is None:
        y_out = torch.empty((N, M), dtype=torch.float32, device=A.device)
    _need(y_out, "y_out", torch.float32, 2)
    _dense(y_out, "y_out")
    idx_out = _idx_out(idx_out, N, C)
    idx_arg = _index_array(idx_out, A, N, D, lda, C, M, True, _act(act), stream)
    st = _lib.lib().maddness_matmul_act_f32(_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C,
                                            _ptr(lut), M, _ptr(col_bias), _act(act), _ptr(y_out),
                                            _ptr(idx_arg), _stream(stream))
    _lib.check("maddness_matmul_act_f32", st)
    return y_out


def build_lut(P, B, stream=None):
    """Table T = P B, 8-bit block-FP quantized; returns (lut int8 [C,16,M], scale [C], offset [C])."""
    _need(P, "P", torch.float32, 3)
    _need(B, "B", torch.float32, 2)
    _dense(P, "P")
    _dense(B, "B")
    C, k, D = P.shape
    if k != K or B.shape[0] != D:
        raise ValueError("P must be [C,16,D] and B [D,M]")
    M = B.shape[1]
    lut = torch.empty((C, K, M), dtype=torch.int8, device=P.device)
    scale = torch.empty((C,), dtype=torch.float32, device=P.device)
    offset = torch.empty((C,), dtype=torch.float32, device=P.device)
    st = _lib.lib().maddness_build_lut(_ptr(P), _ptr(B), C, D, M, _ptr(lut), _ptr(scale),
                                       _ptr(offset), _stream(stream))
    _lib.check("maddness_build_lut", st)
    return lut, scale, offset


def build_lut_shared(P, B, stream=None):
    """build_lut with one block exponent shared by every codebook (for lut_accumulate_avg)."""
    _need(P, "P", torch.float32, 3)
    _need(B, "B", torch.float32, 2)
    _dense(P, "P")
    _dense(B, "B")
    C, k, D = P.shape
    if k != K or B.shape[0] != D:
        raise ValueError("P must be [C,16,D] and B [D,M]")
    M = B.shape[1]
    lut = torch.empty((C, K, M), dtype=torch.int8, device=P.device)
    scale = torch.empty((C,), dtype=torch.float32, device=P.device)
    offset = torch.empty((C,), dtype=torch.float32, device=P.device)
    st = _lib.lib().maddness_build_lut_shared(_ptr(P), _ptr(B), C, D, M, _ptr(lut), _ptr(scale),
                                              _ptr(offset), _stream(stream))
    _lib.check("maddness_build_lut_shared", st)
    return lut, scale, offset


def build_lut_f32(P, B, stream=None):
    """Table T = P B rounded to fp32; returns lut [C,16,M]."""
    _need(P, "P", torch.float32, 3)
    _need(B, "B", torch.float32, 2)
    _dense(P, "P")
    _dense(B, "B")
    C, k, D = P.shape
    if k != K or B.shape[0] != D:
        raise ValueError("P must be [C,16,D] and B [D,M]")
    M = B.shape[1]
    lut = torch.empty((C, K, M), dtype=torch.float32, device=P.device)
    st = _lib.lib().maddness_build_lut_f32(_ptr(P), _ptr(B), C, D, M, _ptr(lut), _stream(stream))
    _lib.check("maddness_build_lut_f32", st)
    return lut


def version() -> int:
    return int(_lib.lib().maddness_version())


class PreparedCall:
    """One C-ABI call with its arguments validated and marshalled once.

    Calling the object issues the same launch again on the stream captured
    when it was prepared (no checks, no allocation, no Python-side work
    beyond the ctypes call), for serving loops and benchmarks.  The tensors
    it was prepared with must stay alive and keep their storage.
    """

    def __init__(self, name, args, keep, outputs):
        self._fn = getattr(_lib.lib(), name)
        self._name = name
        self._args = args
        self._keep = keep          # tensors whose storage the pointers refer to
        self.outputs = outputs

    def __call__(self):
        st = self._fn(*self._args)
        if st:
            _lib.check(self._name, st)
        return self.outputs


def prepare_matmul_f32(A, split_dims, thresholds, lut, y_out=None, idx_out=None, stream=None, validate=False):
    """Prepared maddness_matmul_f32; ``call()`` returns (y, idx or None)."""
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    _need(lut, "lut", torch.float32, 3)
    _dense(lut, "lut")
    C2, M = lut.shape[0], lut.shape[2]
    if lut.shape[1] != K:
        raise ValueError("lut must be [C,16,M]")
    if C2 != C:
        raise ValueError("lut codebooks differ from the trees'")
    if validate:
        _validate_trees(split_dims, D)
    if y_out is None:
        y_out = torch.empty((N, M), dtype=torch.float32, device=A.device)
    _need(y_out, "y_out", torch.float32, 2)
    _dense(y_out, "y_out")
    idx_out = _idx_out(idx_out, N, C)
    idx_arg = _index_array(idx_out, A, N, D, lda, C, M, True, 0, stream)
    args = (_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C, _ptr(lut), M, _ptr(y_out),
            _ptr(idx_arg), _stream(stream))
    keep = (A, split_dims, thresholds, lut, y_out, idx_arg)
    return PreparedCall("maddness_matmul_f32", args, keep, (y_out, idx_out))


def prepare_matmul(A, split_dims, thresholds, lut, scale, offset, y_out=None, acc_out=None,
                   idx_out=None, stream=None, validate=False):
    """Prepared maddness_matmul; ``call()`` returns (y, acc or None, idx or None)."""
    N, D, lda = _rows(A)
    C = _tree_args(split_dims, thresholds)
    C2, M = _lut_i8(lut, scale, offset)
    if C2 != C:
        raise ValueError("lut codebooks differ from the trees'")
    if validate:
        _validate_trees(split_dims, D)
        _validate_scales(scale)
    if y_out is None:
        y_out = torch.empty((N, M), dtype=torch.float32, device=A.device)
    _need(y_out, "y_out", torch.float32, 2)
    _dense(y_out, "y_out")
    idx_out = _idx_out(idx_out, N, C)
    idx_arg = _index_array(idx_out, A, N, D, lda, C, M, False, 0, stream)
    args = (_ptr(A), N, D, lda, _ptr(split_dims), _ptr(thresholds), C, _ptr(lut), _ptr(scale),
            _ptr(offset), M, _ptr(y_out), _ptr(acc_out), _ptr(idx_arg), _stream(stream))
    keep = (A, split_dims, thresholds, lut, scale, offset, y_out, acc_out, idx_arg)
    return PreparedCall("maddness_matmul", args, keep, (y_out, acc_out, idx_out))


def quantize_lut(T, shared=False, stream=None):
    """8-bit block floating point quantization of a given float64 table
    [C,16,M] (e.g. a fitted one); returns (lut, scale, offset)."""
    _need(T, "T", torch.float64, 3)
    _dense(T, "T")
    C, k, M = T.shape
    if k != K:
        raise ValueError("T must be [C,16,M]")
    lut = torch.empty((C, K, M), dtype=torch.int8, device=T.device)
    scale = torch.empty((C,), dtype=torch.float32, device=T.device)
    offset = torch.empty((C,), dtype=torch.float32, device=T.device)
    st = _lib.lib().maddness_quantize_lut(_ptr(T), C, M, 1 if shared else 0, _ptr(lut), _ptr(scale), _ptr(offset),
                                          _stream(stream))
    _lib.check("maddness_quantize_lut", st)
    return lut, scale, offset


def _fit_inputs(idx, Y):
    _need(idx, "idx", torch.uint8, 2)
    _dense(idx, "idx")
    _need(Y, "Y", torch.float32, 2)
    _dense(Y, "Y")
    if Y.shape[0] != idx.shape[0]:
        raise ValueError("Y must have one row per index row")
    return idx.shape[0], idx.shape[1], Y.shape[1]


def encoder_gram(idx, stream=None):
    """H = G^T G of the one-hot encoder output: int32 [16C, 16C] counts."""
    _need(idx, "idx", torch.uint8, 2)
    _dense(idx, "idx")
    N, C = idx.shape
    H = torch.empty((C * K, C * K), dtype=torch.int32, device=idx.device)
    st = _lib.lib().maddness_encoder_gram(_ptr(idx), N, C, _ptr(H), _stream(stream))
    _lib.check("maddness_encoder_gram", st)
    return H


def _workspace(workspace, need, device, stream):
    """A 256-byte aligned pointer into ``workspace`` (allocated when None)."""
    if workspace is None:
        workspace = torch.empty((need + 256,), dtype=torch.uint8, device=device)
        if stream is not None:
            workspace.record_stream(stream)   # freed only after the work queued on `stream`
    base = workspace.data_ptr()
    off = (-base) % 256
    if workspace.numel() - off < need:
        raise ValueError(f"workspace must hold {need} bytes at a 256-byte aligned address")
    return workspace, ctypes.c_void_p(base + off)


def encoder_scatter(idx, Y, workspace=None, stream=None):
    """R = G^T Y: float64 [16C, M], each entry summed over its rows in order."""
    N, C, M = _fit_inputs(idx, Y)
    need = int(_lib.lib().maddness_encoder_scatter_workspace_bytes(N, C))
    if need < 0:
        _lib.check("maddness_encoder_scatter", _lib.EUNSUPPORTED)
    workspace, wp = _workspace(workspace, need, idx.device, stream)
    R = torch.empty((C * K, M), dtype=torch.float64, device=idx.device)
    st = _lib.lib().maddness_encoder_scatter(_ptr(idx), N, C, _ptr(Y), M, _ptr(R), wp, need, _stream(stream))
    _lib.check("maddness_encoder_scatter", st)
    return R


def fit_lut_ridge(idx, Y, T0, lam, workspace=None, stream=None):
    """Model-aware table fit (Eq. 3, affine output): the float64 table
    [C,16,M] minimising ||Y - G T||^2 + lam ||T - T0||^2.  ``workspace``: an
    optional preallocated uint8 device tensor of at least
    fit_lut_workspace_bytes(N, C) bytes (+ up to 255 for alignment)."""
    N, C, M = _fit_inputs(idx, Y)
    _need(T0, "T0", torch.float32, 3)
    _dense(T0, "T0")
    if tuple(T0.shape) != (C, K, M):
        raise ValueError("T0 must be [C,16,M]")
    need = int(_lib.lib().maddness_fit_lut_workspace_bytes(N, C))
    if need < 0:
        _lib.check("maddness_fit_lut_ridge", _lib.EUNSUPPORTED)
    workspace, wp = _workspace(workspace, need, idx.device, stream)
    T = torch.empty((C, K, M), dtype=torch.float64, device=idx.device)
    st = _lib.lib().maddness_fit_lut_ridge(_ptr(idx), N, C, _ptr(Y), M, _ptr(T0), float(lam), _ptr(T),
                                           wp, need, _stream(stream))
    _lib.check("maddness_fit_lut_ridge", st)
    return T


def fit_lut_workspace_bytes(N: int, C: int) -> int:
    """Device bytes fit_lut_ridge needs as workspace for N training rows and C codebooks."""
    n = int(_lib.lib().maddness_fit_lut_workspace_bytes(N, C))
    if n < 0:
        _lib.check("maddness_fit_lut_workspace_bytes", _lib.EUNSUPPORTED)
    return n


def fit_lut_gd(idx, Y, T0, act, lam, eta, iters, col_bias=None, workspace=None, stream=None):
    """Model-aware table fit (Eq. 3) with a nonlinear output by gradient
    descent from T0: act "relu" (squared error after bias + ReLU),
    "softmax" / "softmax_kld" (KL divergence between row softmaxes) or
    "softmax_sqerr" (squared error between row softmaxes); float64 [C,16,M]."""
    N, C, M = _fit_inputs(idx, Y)
    _need(T0, "T0", torch.float32, 3)
    _dense(T0, "T0")
    if tuple(T0.shape) != (C, K, M):
        raise ValueError("T0 must be [C,16,M]")
    if isinstance(act, str) and act not in FIT:
        raise ValueError(f"act must be one of {sorted(FIT)}")
    code = FIT[act] if isinstance(act, str) else int(act)
    if col_bias is not None:
        _need(col_bias, "col_bias", torch.float32, 1)
        _dense(col_bias, "col_bias")
        if col_bias.shape[0] != M:
            raise ValueError("col_bias must be [M]")
    need = int(_lib.lib().maddness_fit_lut_gd_workspace_bytes(N, C, M))
    if need < 0:
        _lib.check("maddness_fit_lut_gd", _lib.EUNSUPPORTED)
    workspace, wp = _workspace(workspace, need, idx.device, stream)
    T = torch.empty((C, K, M), dtype=torch.float64, device=idx.device)
    st = _lib.lib().maddness_fit_lut_gd(_ptr(idx), N, C, _ptr(Y), M, _ptr(col_bias), int(code), _ptr(T0), float(lam),
                                        float(eta), int(iters), _ptr(T), wp, need, _stream(stream))
    _lib.check("maddness_fit_lut_gd", st)
    return T


def fit_lut_gd_workspace_bytes(N: int, C: int, M: int) -> int:
    """Device bytes fit_lut_gd needs as workspace."""
    n = int(_lib.lib().maddness_fit_lut_gd_workspace_bytes(N, C, M))
    if n < 0:
        _lib.check("maddness_fit_lut_gd_workspace_bytes", _lib.EUNSUPPORTED)
    return n


# ------------------------------------------------- the output layer's operators

# element types (MADDNESS_F32, _BF16, _F16)
DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _typed(t, name: str, dtypes, ndim: int) -> int:
    """Checks a device tensor of one of these types; returns the ABI's code."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be one of {', '.join(str(d) for d in dtypes)}, got {t.dtype}")
    _need(t, name, t.dtype, ndim)
    return DTYPE[t.dtype]


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} must be on {device}, got {t.device}")


def _plain_call(name, *args):
    """One of the natively marshalled calls on the current device and stream;
    None when the arguments are not its plain valid case (the caller then goes
    through its own checks), or there is no native marshalling."""
    global _calls
    if _calls is None:
        _calls = _lib.calls() or False
    if not _calls:
        return None
    device = torch._C._cuda_getDevice()
    return getattr(_calls, name)(*args, device, torch._C._cuda_getCurrentRawStream(device))


_calls = None


def _on_gpu(t) -> bool:
    return type(t) is torch.Tensor and t.is_cuda


@contextlib.contextmanager
def _device(device):
    """The device of the call's tensors as the current one."""
    if device.index == torch.cuda.current_device():
        yield
    else:
        with torch.cuda.device(device):
            yield


def _row_stride(A) -> int:
    """Elements between A's rows, whose columns must be dense."""
    N, D = A.shape
    if D > 1 and N > 0 and A.stride(1) != 1:
        raise ValueError("A must have unit column stride")
    if N > 1 and A.stride(0) < D:
        raise ValueError("A's rows must not overlap")
    return A.stride(0) if N > 1 else D


def _scratch(workspace, need: int, device, stream):
    """_workspace of a caller's tensor checked for type and device."""
    if workspace is not None:
        _need(workspace, "workspace", torch.uint8, 1)
        _dense(workspace, "workspace")
        _same_device(device, workspace=workspace)
    return _workspace(workspace, need, device, stream)


def _output(t, name: str, shape, dtype, device):
    """The caller's output tensor checked, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _need(t, name, dtype, len(shape))
    _dense(t, name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    _same_device(device, **{name: t})
    return t


class W4Weights(NamedTuple):
    """4-bit block floating point weights of a layer [D, M] in the packed
    layout of include/maddness.h: codes uint8 [ceil(M / 16), ceil(D / 128), 64,
    16] and exps uint8 [ceil(M / 16), ceil(D / 128), 16, 4]."""
    codes: torch.Tensor
    exps: torch.Tensor
    D: int
    M: int


def _w4(w):
    if not isinstance(w, W4Weights):
        raise TypeError("weights must be W4Weights (quantize_w4 makes them)")
    _need(w.codes, "codes", torch.uint8, 4)
    _need(w.exps, "exps", torch.uint8, 4)
    _dense(w.codes, "codes")
    _dense(w.exps, "exps")
    D, M = int(w.D), int(w.M)
    if D <= 0 or M <= 0:
        raise ValueError("D and M must be positive")
    blocks = ((M + 15) // 16, (D + 127) // 128)
    if tuple(w.codes.shape) != blocks + (64, 16) or tuple(w.exps.shape) != blocks + (16, 4):
        raise ValueError(f"weights of [{D}, {M}] have codes {list(blocks + (64, 16))} and exps {list(blocks + (16, 4))}, "
                         f"got {list(w.codes.shape)} and {list(w.exps.shape)}")
    _same_device(w.codes.device, exps=w.exps)
    return D, M


def quantize_w4(B, stream=None) -> W4Weights:
    """4-bit block floating point weights of B [D, M] (fp32, bf16 or fp16, any
    strides); see maddness_quantize_w4."""
    if stream is None and _on_gpu(B):
        r = _plain_call("quantize", B)
        if r is not None:
            return W4Weights(*r, *B.shape)
    code = _typed(B, "B", (torch.float32, torch.bfloat16, torch.float16), 2)
    D, M = B.shape
    if D == 0 or M == 0:
        raise ValueError("B must not be empty")
    blocks = ((M + 15) // 16, (D + 127) // 128)
    with _device(B.device):
        codes = torch.empty(blocks + (64, 16), dtype=torch.uint8, device=B.device)
        exps = torch.empty(blocks + (16, 4), dtype=torch.uint8, device=B.device)
        st = _lib.lib().maddness_quantize_w4(_ptr(B), code, D, M, B.stride(0), B.stride(1), _ptr(codes), _ptr(exps),
                                             _stream(stream))
    _lib.check("maddness_quantize_w4", st)
    return W4Weights(codes, exps, D, M)


def dequantize_w4(w: W4Weights, dtype=torch.bfloat16, out=None, stream=None):
    """The weights [D, M] that the codes stand for, as bf16 or fp32 (both exact)."""
    if stream is None and out is None and type(w) is W4Weights and _on_gpu(w.codes):
        r = _plain_call("dequantize", w.codes, w.exps, w.D, w.M, DTYPE.get(dtype, -1))
        if r is not None:
            return r
    D, M = _w4(w)
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"dtype must be torch.float32 or torch.bfloat16, got {dtype}")
    with _device(w.codes.device):
        out = _output(out, "out", (D, M), dtype, w.codes.device)
        st = _lib.lib().maddness_dequantize_w4(_ptr(w.codes), _ptr(w.exps), D, M, _ptr(out), DTYPE[dtype], _stream(stream))
    _lib.check("maddness_dequantize_w4", st)
    return out


def matmul_w4(A, w: W4Weights, col_bias=None, act=None, out_dtype=None, y_out=None, workspace=None, stream=None):
    """Layer with 4-bit weights, sigma(A W + col_bias); returns y [N, M].

    A [N, D] fp32, bf16 or fp16 with dense columns.  act "none" (no bias),
    "bias", "relu" or "softmax"; None: "bias" where one is given.  y has A's
    dtype, or out_dtype torch.float32, which a softmax always gives.
    ``workspace``: an optional uint8 device tensor of at least
    matmul_w4_workspace_bytes(A, M) bytes (+ up to 255 for alignment), used for
    many rows; allocated when None."""
    if act is None:
        act = "none" if col_bias is None else "bias"
    if stream is None and y_out is None and workspace is None and _on_gpu(A) and type(w) is W4Weights:
        r = _plain_call("w4", A, w.codes, w.exps, w.D, w.M, col_bias, ACT.get(act, -1) if isinstance(act, str) else -1,
                        -1 if out_dtype is None else DTYPE.get(out_dtype, 9))
        if r is not None:
            return r
    code = _typed(A, "A", (torch.float32, torch.bfloat16, torch.float16), 2)
    D, M = _w4(w)
    N = A.shape[0]
    if A.shape[1] != D:
        raise ValueError(f"A must have the weights' {D} columns, got {A.shape[1]}")
    lda = _row_stride(A)
    col_bias = _col_bias(col_bias, M)
    _same_device(A.device, weights=w.codes, col_bias=col_bias)
    a = _act(act)
    if out_dtype is None:
        out_dtype = y_out.dtype if y_out is not None else torch.float32 if a == ACT["softmax"] else A.dtype
    if out_dtype not in (A.dtype, torch.float32):
        raise TypeError(f"out_dtype must be {A.dtype} or torch.float32, got {out_dtype}")
    if a == ACT["softmax"] and out_dtype != torch.float32:
        raise TypeError("a softmax gives torch.float32")
    with _device(A.device):
        y_out = _output(y_out, "y_out", (N, M), out_dtype, A.device)
        need, wp = int(_lib.lib().maddness_matmul_w4_workspace_bytes(_ptr(A), code, N, D, lda, M)), None
        if need > 0:
            workspace, wp = _scratch(workspace, need, A.device, stream)
        st = _lib.lib().maddness_matmul_w4(_ptr(A), code, N, D, lda, _ptr(w.codes), _ptr(w.exps), M, _ptr(col_bias), a,
                                           _ptr(y_out), DTYPE[out_dtype], wp, need, _stream(stream))
    _lib.check("maddness_matmul_w4", st)
    return y_out


def matmul_w4_workspace_bytes(A, M: int) -> int:
    """Device bytes of workspace that matmul_w4 uses for this A (its shape,
    type and alignment) and M outputs; 0 where it uses none."""
    code = _typed(A, "A", (torch.float32, torch.bfloat16, torch.float16), 2)
    n = int(_lib.lib().maddness_matmul_w4_workspace_bytes(_ptr(A), code, A.shape[0], A.shape[1], _row_stride(A), M))
    if n < 0:
        _lib.check("maddness_matmul_w4_workspace_bytes", _lib.EINVAL)
    return n


def _xent_inputs(A, B, target, col_bias):
    code = _typed(A, "A", (torch.float32, torch.bfloat16), 2)
    _need(B, "B", A.dtype, 2)
    _need(target, "target", torch.int64, 1)
    _dense(target, "target")
    N, D = A.shape
    M = B.shape[1]
    if D == 0 or M == 0:
        raise ValueError("A and B must have columns")
    if B.shape[0] != D or target.shape[0] != N:
        raise ValueError(f"A [N, D], B [D, M] and target [N] do not fit: {list(A.shape)}, {list(B.shape)}, {list(target.shape)}")
    if not B.is_contiguous() and not B.t().is_contiguous():
        raise ValueError("B must be contiguous, or the transpose of a contiguous tensor")
    first = 0 if B.is_contiguous() else 1
    col_bias = _col_bias(col_bias, M)
    _same_device(A.device, B=B, target=target, col_bias=col_bias)
    return code, N, D, M, _row_stride(A), first, col_bias


def linear_xent(A, B, target, col_bias=None, loss_out=None, lse_out=None, workspace=None, stream=None):
    """Softmax cross entropy of the output layer A B + col_bias without keeping
    the logits; returns (loss [N], lse [N]) in fp32.

    A [N, D] and B [D, M] fp32 or bf16 (B contiguous, or the transpose of a
    contiguous [M, D]); target [N] int64, outside [0, M) for rows without a
    loss.  ``workspace``: an optional uint8 device tensor of at least
    linear_xent_workspace_bytes(N, D, M, A.dtype) bytes (+ up to 255 for
    alignment)."""
    if stream is None and loss_out is None and lse_out is None and workspace is None and _on_gpu(A):
        r = _plain_call("xent", A, B, target, col_bias)
        if r is not None:
            return r
    code, N, D, M, lda, first, col_bias = _xent_inputs(A, B, target, col_bias)
    with _device(A.device):
        loss_out = _output(loss_out, "loss_out", (N,), torch.float32, A.device)
        lse_out = _output(lse_out, "lse_out", (N,), torch.float32, A.device)
        need = linear_xent_workspace_bytes(N, D, M, A.dtype)
        workspace, wp = _scratch(workspace, need, A.device, stream)
        st = _lib.lib().maddness_linear_xent(_ptr(A), code, N, D, lda, _ptr(B), M, first, _ptr(col_bias), _ptr(target),
                                             _ptr(loss_out), _ptr(lse_out), wp, need, _stream(stream))
    _lib.check("maddness_linear_xent", st)
    return loss_out, lse_out


def linear_xent_grad(A, B, target, lse, grad_loss, col_bias=None, dA_out=None, dB_out=None, dbias_out=None, workspace=None,
                     stream=None):
    """The gradient of (grad_loss * loss).sum(): returns (dA [N, D], dB [D, M],
    dbias [M]); dA and dB in A's dtype, dB laid out like B, dbias fp32.

    lse [N] as linear_xent gave it for the same A, B, target and col_bias;
    grad_loss [N] fp32.  ``workspace``: an optional uint8 device tensor of at
    least linear_xent_grad_workspace_bytes(N, D, M, A.dtype) bytes (+ up to 255
    for alignment)."""
    if stream is None and dA_out is None and dB_out is None and dbias_out is None and workspace is None and _on_gpu(A):
        r = _plain_call("xent_grad", A, B, target, col_bias, lse, grad_loss)
        if r is not None:
            return r
    code, N, D, M, lda, first, col_bias = _xent_inputs(A, B, target, col_bias)
    for t, name in ((lse, "lse"), (grad_loss, "grad_loss")):
        _need(t, name, torch.float32, 1)
        _dense(t, name)
        if t.shape[0] != N:
            raise ValueError(f"{name} must be [N]")
    _same_device(A.device, lse=lse, grad_loss=grad_loss)
    with _device(A.device):
        dA_out = _output(dA_out, "dA_out", (N, D), A.dtype, A.device)
        if dB_out is not None and first:
            _need(dB_out, "dB_out", A.dtype, 2)
            _output(dB_out.t(), "dB_out's transpose", (M, D), A.dtype, A.device)
        elif first:
            dB_out = torch.empty((M, D), dtype=A.dtype, device=A.device).t()
        else:
            dB_out = _output(dB_out, "dB_out", (D, M), A.dtype, A.device)
        dbias_out = _output(dbias_out, "dbias_out", (M,), torch.float32, A.device)
        need = linear_xent_grad_workspace_bytes(N, D, M, A.dtype)
        workspace, wp = _scratch(workspace, need, A.device, stream)
        st = _lib.lib().maddness_linear_xent_grad(_ptr(A), code, N, D, lda, _ptr(B), M, first, _ptr(col_bias), _ptr(target),
                                                  _ptr(lse), _ptr(grad_loss), _ptr(dA_out), _ptr(dB_out), _ptr(dbias_out),
                                                  wp, need, _stream(stream))
    _lib.check("maddness_linear_xent_grad", st)
    return dA_out, dB_out, dbias_out


def _xent_bytes(fn, N, D, M, dtype) -> int:
    n = int(getattr(_lib.lib(), fn)(N, D, M, DTYPE.get(dtype, -1)))
    if n < 0:
        _lib.check(fn, _lib.EUNSUPPORTED)
    return n


def linear_xent_workspace_bytes(N: int, D: int, M: int, dtype=torch.float32) -> int:
    """Device bytes linear_xent needs as workspace."""
    return _xent_bytes("maddness_linear_xent_workspace_bytes", N, D, M, dtype)


def linear_xent_grad_workspace_bytes(N: int, D: int, M: int, dtype=torch.float32) -> int:
    """Device bytes linear_xent_grad needs as workspace."""
    return _xent_bytes("maddness_linear_xent_grad_workspace_bytes", N, D, M, dtype)
