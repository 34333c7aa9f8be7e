"""The experts' matrix products on their own: grouped by expert with ragged row counts, their gradients,
and the same in 8-bit floating point (e4m3) with a scale for each block of 128.

As in binding.py the functions carry the C entry points' names, check and marshal their arguments, and
allocate what the caller does not pass. Rows and groups are a PathTable's: offsets [n+1] int32 (its
expert_offsets), row_token [R] int32 (row of x behind each row) and row_of [T, k] int32. Without offsets
there is one group and w may be [N, K]. Tensors must be contiguous, on the current device; 8-bit values
are torch.float8_e4m3fn, their scales float32. Autograd does not record these calls, whatever their inputs
require: a backward pass makes the gradients' calls itself."""
from __future__ import annotations

from typing import Optional

import torch

from .binding import OP_GROUPED_DW, OP_GROUPED_DX, PCM_BF16, PCM_F32, _check, _on, lib, workspace_bytes

_CODES = {torch.float32: PCM_F32, torch.bfloat16: PCM_BF16}
_E4M3 = torch.float8_e4m3fn


# Small calls are bound by the host: pointers go as plain integers (None for none), and the current stream's
# handle comes without a Stream object around it (a call of 12.6 us takes 8.5 that way).
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream_on(stream, device):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    if stream.device != device:
        raise ValueError(f"stream must be on {device}")
    return stream.cuda_stream


def _blocks(size: int) -> int:
    return (size + 127) // 128


def _code(dtype: torch.dtype) -> int:
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}: float32 or bfloat16")
    return code


def _operand(t: torch.Tensor, what: str, dtype=None, shape=None, device: Optional[torch.device] = None):
    """Checks a tensor the kernels address: device, layout, and dtype and shape where they are given."""
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous device tensor")
    if device is None:
        if t.device.index != torch.cuda.current_device():
            raise ValueError(f"{what} must be on the current device")
    elif t.device != device:
        raise ValueError(f"{what} must be on {device}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")


# The C entry points take widths and numbers of groups and slots in 32 bits; ctypes would cut larger ones.
_INT_MAX = 2 ** 31 - 1


def _too_wide(what: str):
    raise ValueError(f"{what}: a size does not fit in 32 bits")


def _weights(w: torch.Tensor, offsets: Optional[torch.Tensor]):
    """(n, N, K) of w [n, N, K], or of a plain product's w [N, K]."""
    if w.dim() == 2 and offsets is None:
        n, (N, K) = 1, w.shape
    elif w.dim() != 3:
        raise ValueError("w must have shape [n, N, K]")
    else:
        n, N, K = w.shape
    if n > _INT_MAX or N > _INT_MAX or K > _INT_MAX:
        _too_wide("w")
    return n, N, K


def _rows(x_rows: int, n: int, offsets, row_token, device) -> int:
    """The number of rows: row_token's, or those of x."""
    if offsets is not None:
        _operand(offsets, "offsets", torch.int32, (n + 1,), device)
    elif n != 1 or row_token is not None:
        raise ValueError("several groups, or gathered rows, need offsets")
    if row_token is None:
        return x_rows
    if row_token.dim() != 1:
        raise ValueError("row_token must have shape [R]")
    _operand(row_token, "row_token", torch.int32, None, device)
    return row_token.shape[0]


def _matrix(t: torch.Tensor, what: str):
    if t.dim() != 2:
        raise ValueError(f"{what} must have two dimensions")
    if t.shape[1] > _INT_MAX:
        _too_wide(what)
    return t.shape


def _out(t, shape, dtype, device, what, stream):
    if t is None:
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=device)
        with _on(stream):
            return torch.empty(shape, dtype=dtype, device=device)
    _operand(t, what, dtype, shape, device)
    return t


def _workspace(ws, nbytes: int, device, stream):
    if not nbytes:
        return None
    return _out(ws, (nbytes,) if ws is None else ws.shape, torch.uint8, device, "ws", stream)


def pcm_grouped_gemm(x: torch.Tensor, w: torch.Tensor, offsets=None, row_token=None, y=None,
                     out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """y[r] = x[row_token[r]] w[e]^T for the rows r of group e (row r of x without row_token).
    out_dtype: x's, or float32. Rows from offsets[n] on are not written."""
    T, K = _matrix(x, "x")
    n, N, _ = _weights(w, offsets)
    _operand(x, "x")
    dev = x.device
    _operand(w, "w", x.dtype, (n, N, K) if w.dim() == 3 else (N, K), dev)
    R = _rows(T, n, offsets, row_token, dev)
    out = y.dtype if y is not None and out_dtype is None else out_dtype or x.dtype
    y = _out(y, (R, N), out, dev, "y", stream)
    status = lib().pcm_grouped_gemm(_code(x.dtype), _code(out), _ptr(x), _ptr(w), _ptr(offsets), _ptr(row_token), T, R,
                                  K, N, n, _ptr(y), _stream_on(stream, dev))
    if status:
        _check(status)
    return y


def pcm_grouped_gemm_dx(dy: torch.Tensor, w: torch.Tensor, offsets=None, row_of=None, dx=None,
                        out_dtype: Optional[torch.dtype] = None, ws: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """The gradient by x: dy[r] w[e] for every row, or, with row_of [T, k] (outside the groups' rows: none),
    its sum over the rows of each token. ws: workspace_bytes(OP_GROUPED_DX, T, K, 0, n, k, dtype) bytes, with row_of."""
    R, N = _matrix(dy, "dy")
    n, _, K = _weights(w, offsets)
    T, k = (R, 1) if row_of is None else _matrix(row_of, "row_of")
    _operand(dy, "dy")
    dev = dy.device
    _operand(w, "w", dy.dtype, (n, N, K) if w.dim() == 3 else (N, K), dev)
    _rows(R, n, offsets, None, dev)
    code = _code(dy.dtype)
    out = dx.dtype if dx is not None and out_dtype is None else out_dtype or dy.dtype
    nbytes = 0
    if row_of is not None:
        _operand(row_of, "row_of", torch.int32, None, dev)
        nbytes = workspace_bytes(OP_GROUPED_DX, T, K, 0, n, k, code)
    ws = _workspace(ws, nbytes, dev, stream)
    dx = _out(dx, (T, K), out, dev, "dx", stream)
    status = lib().pcm_grouped_gemm_dx(code, _code(out), _ptr(dy), _ptr(w), _ptr(offsets), _ptr(row_of), T, k, R, K, N, n,
                                     _ptr(dx), _ptr(ws), ws.numel() if nbytes else 0,
                                     _stream_on(stream, dev))
    if status:
        _check(status)
    return dx


def pcm_grouped_gemm_dw(x: torch.Tensor, dy: torch.Tensor, offsets=None, row_token=None, dw=None,
                        out_dtype: Optional[torch.dtype] = None, accumulate: bool = False,
                        ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The gradient by w, [n, N, K] ([N, K] without offsets): the sum of dy[r]^T x[row_token[r]] over the rows
    of each group, zero for an empty one. accumulate adds into dw, which is then float32.
    ws: workspace_bytes(OP_GROUPED_DW, R, K, N, n, 1, dtype) bytes."""
    T, K = _matrix(x, "x")
    R, N = _matrix(dy, "dy")
    _operand(x, "x")
    dev = x.device
    _operand(dy, "dy", x.dtype, None, dev)
    if offsets is not None and (offsets.dim() != 1 or offsets.shape[0] < 2):
        raise ValueError("offsets must have shape [n + 1]")
    n = 1 if offsets is None else offsets.shape[0] - 1
    if _rows(T, n, offsets, row_token, dev) != R:
        raise ValueError("dy must have a row for each row")
    if accumulate and dw is None:
        raise ValueError("accumulate needs dw")
    out = dw.dtype if dw is not None and out_dtype is None else out_dtype or x.dtype
    dw = _out(dw, (n, N, K) if offsets is not None or (dw is not None and dw.dim() == 3) else (N, K), out, dev, "dw", stream)
    code = _code(x.dtype)
    nbytes = workspace_bytes(OP_GROUPED_DW, R, K, N, n, 1, code)
    ws = _workspace(ws, nbytes, dev, stream)
    status = lib().pcm_grouped_gemm_dw(code, _code(out), _ptr(x), _ptr(dy), _ptr(offsets), _ptr(row_token), T, R, K, N, n,
                                       _ptr(dw), int(bool(accumulate)), _ptr(ws), ws.numel() if nbytes else 0,
                                       _stream_on(stream, dev))
    if status:
        _check(status)
    return dw


def _count(count, device):
    if count is not None:
        if count.dim() > 1 or count.numel() != 1:
            raise ValueError("count must be one number")
        _operand(count, "count", torch.int32, None, device)


def _quant_rows(name, x, K, count, q, scale, stream):
    R = x.shape[0]
    _operand(x, "x")
    dev = x.device
    _count(count, dev)
    q = _out(q, (R, K), _E4M3, dev, "q", stream)
    scale = _out(scale, (R, _blocks(K)), torch.float32, dev, "scale", stream)
    status = getattr(lib(), name)(_code(x.dtype), _ptr(x), _ptr(count), R, K, _ptr(q), _ptr(scale), _stream_on(stream, dev))
    if status:
        _check(status)
    return q, scale


def pcm_quant_fp8_rows(x: torch.Tensor, count=None, q=None, scale=None, stream=None):
    """(q, scale): the rows of x [R, K] in 8 bits, with a scale for each block of 128 columns. count: one
    int32 on the device (such as offsets[-1]); rows from there on are left as they were."""
    _, K = _matrix(x, "x")
    return _quant_rows("pcm_quant_fp8_rows", x, K, count, q, scale, stream)


def pcm_swiglu_quant_fp8(gate_up: torch.Tensor, count=None, q=None, scale=None, stream=None):
    """pcm_quant_fp8_rows of SiLU(gate) * up; gate_up [R, 2F] holds a row's gate values before its up values."""
    if gate_up.dim() != 2 or gate_up.shape[1] % 2:
        raise ValueError("gate_up must have two dimensions and an even number of columns")
    K2 = gate_up.shape[1]
    if K2 // 2 > _INT_MAX:
        _too_wide("gate_up")
    return _quant_rows("pcm_swiglu_quant_fp8", gate_up, K2 // 2, count, q, scale, stream)


def pcm_quant_fp8_weights(w: torch.Tensor, transpose: bool = False, q=None, scale=None, q_t=None, scale_t=None,
                          stream=None):
    """(q, scale): w [n, N, K] (or [N, K]) in 8 bits, with a scale for each 128 x 128 block; with `transpose`
    also (q_t, scale_t), the same codes and scales of every w^T (for the gradient by the input)."""
    if w.dim() not in (2, 3):
        raise ValueError("w must have shape [n, N, K] or [N, K]")
    if max(w.shape) > _INT_MAX:
        _too_wide("w")
    _operand(w, "w")
    dev, lead = w.device, tuple(w.shape[:-2])
    n, (N, K) = lead[0] if lead else 1, w.shape[-2:]
    q = _out(q, lead + (N, K), _E4M3, dev, "q", stream)
    scale = _out(scale, lead + (_blocks(N), _blocks(K)), torch.float32, dev, "scale", stream)
    if transpose:
        q_t = _out(q_t, lead + (K, N), _E4M3, dev, "q_t", stream)
        scale_t = _out(scale_t, lead + (_blocks(K), _blocks(N)), torch.float32, dev, "scale_t", stream)
    elif q_t is not None or scale_t is not None:
        raise ValueError("q_t and scale_t need transpose")
    status = lib().pcm_quant_fp8_weights(_code(w.dtype), _ptr(w), n, N, K, _ptr(q), _ptr(scale), _ptr(q_t), _ptr(scale_t),
                                       _stream_on(stream, dev))
    if status:
        _check(status)
    return (q, scale, q_t, scale_t) if transpose else (q, scale)


def pcm_grouped_gemm_fp8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, offsets=None,
                         row_token=None, y=None, out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """pcm_grouped_gemm of 8-bit operands and their scales (pcm_quant_fp8_rows, pcm_quant_fp8_weights).
    out_dtype: float32, with exact products of codes, or bfloat16 (the default), with those of the 8-bit matrix
    cores, which cut a product below 2^-13 of the largest among its neighbours: 1.3e-5 of the result's norm on
    normal values (the rounding to bfloat16: 1.7e-3). x_scale * w_scale has to be a normal float32 number."""
    T, K = _matrix(x, "x")
    n, N, _ = _weights(w, offsets)
    _operand(x, "x", _E4M3)
    dev = x.device
    lead = (n,) if w.dim() == 3 else ()
    _operand(w, "w", _E4M3, lead + (N, K), dev)
    _operand(x_scale, "x_scale", torch.float32, (T, _blocks(K)), dev)
    _operand(w_scale, "w_scale", torch.float32, lead + (_blocks(N), _blocks(K)), dev)
    R = _rows(T, n, offsets, row_token, dev)
    out = y.dtype if y is not None and out_dtype is None else out_dtype or torch.bfloat16
    y = _out(y, (R, N), out, dev, "y", stream)
    status = lib().pcm_grouped_gemm_fp8(_code(out), _ptr(x), _ptr(x_scale), _ptr(w), _ptr(w_scale), _ptr(offsets),
                                      _ptr(row_token), T, R, K, N, n, _ptr(y), _stream_on(stream, dev))
    if status:
        _check(status)
    return y
