"""What a training step does around the experts' products (experts.py): tokens to their experts' rows and back with
weights applied, SwiGLU, the mix along a token's paths, each with its gradient; the router's gradient; the norm over
all gradients and clipping.

As in experts.py the functions carry the C entry points' names, check and marshal their arguments, and allocate what
the caller does not pass. row_of [T, k] int32, offsets [n+1] int32, path_bits [T] int64 and beta [T, k, k] float32 are
a PathTable's (or a ScoredPathTable's src_row_of and tgt_row_of). Tensors are float32 or bfloat16, contiguous, on the
current device and, but for offsets, counts, norms and the gradients of the norm and the clipping, aligned to 16 bytes (a
row_of of some tokens, sliced from a larger one, may not be: it is refused); out_dtype is either type, by default the
input's. Sums are float32, rounded once. Autograd does not record these calls: a backward pass makes the gradients' calls
itself."""
from __future__ import annotations

from array import array
from typing import Optional, Sequence

import torch

from .binding import BETA_SRC_COND, OP_GRAD_NORM, _check, lib, workspace_bytes
from .experts import _CODES, _code, _count, _INT_MAX, _matrix, _operand, _out, _ptr, _stream_on, _too_wide, _workspace

_F32 = torch.float32


def _out_type(given: Optional[torch.Tensor], out_dtype: Optional[torch.dtype], default: torch.dtype) -> torch.dtype:
    return given.dtype if given is not None and out_dtype is None else out_dtype or default


def _table(row_of, what, device, shape=None):
    T, k = _matrix(row_of, what)
    _operand(row_of, what, torch.int32, shape, device)
    return T, k


def _slots(row_of, weights, offsets, device):
    """(T, k, n) of the rows' numbers, with their weights and the groups' bounds."""
    T, k = _table(row_of, "row_of", device)
    if weights is not None:
        _operand(weights, "weights", _F32, (T, k), device)
    n = 1
    if offsets is not None:
        if offsets.dim() != 1 or offsets.shape[0] < 2:
            raise ValueError("offsets must have shape [n + 1]")
        _operand(offsets, "offsets", torch.int32, None, device)
        n = offsets.shape[0] - 1
    return T, k, n


def _row_count(rows: Optional[int], given, T: int, k: int) -> int:
    if given is not None:
        if rows is not None and rows != given.shape[0]:
            raise ValueError(f"the row buffer must have {rows} rows, not {given.shape[0]}")
        return given.shape[0]
    return T * k if rows is None else rows


def pcm_dispatch_rows(x: torch.Tensor, row_of: torch.Tensor, weights=None, offsets=None, rows: Optional[int] = None, y=None,
                      out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """y[row_of[t, a]] = weights[t, a] x[t]; y has `rows` rows (T k by default). Rows of no pair are left as they were
    (in a y that the caller does not pass: undefined). row_of outside the groups' rows: none."""
    T, H = _matrix(x, "x")
    _operand(x, "x")
    dev = x.device
    t, k, n = _slots(row_of, weights, offsets, dev)
    if t != T:
        raise ValueError("row_of must have a row for each token")
    out = _out_type(y, out_dtype, x.dtype)
    R = _row_count(rows, y, T, k)
    y = _out(y, (R, H), out, dev, "y", stream)
    status = lib().pcm_dispatch_rows(_code(x.dtype), _code(out), _ptr(x), _ptr(row_of), _ptr(weights), _ptr(offsets), T, k, R, H,
                                     n, _ptr(y), _stream_on(stream, dev))
    if status:
        _check(status)
    return y


def pcm_dispatch_rows_grad(dy: torch.Tensor, row_of: torch.Tensor, x: Optional[torch.Tensor] = None, weights=None, offsets=None,
                           dx=None, dweights=None, out_dtype: Optional[torch.dtype] = None, stream=None):
    """(dx, dweights) of pcm_dispatch_rows: the sum of weights[t, a] dy[row_of[t, a]] over a token's slots, and, with x, the
    products <dy[row_of[t, a]], x[t]> (None without). x may be of the other type."""
    R, H = _matrix(dy, "dy")
    _operand(dy, "dy")
    dev = dy.device
    T, k, n = _slots(row_of, weights, offsets, dev)
    out = _out_type(dx, out_dtype, dy.dtype)
    dweights = _dots(x, "x", (T, H), None, dweights, (T, k), dev, stream)
    dx = _out(dx, (T, H), out, dev, "dx", stream)
    status = lib().pcm_dispatch_rows_grad(_code(dy.dtype), _code((dy if x is None else x).dtype), _code(out), _ptr(dy), _ptr(x), _ptr(row_of), _ptr(weights),
                                          _ptr(offsets), T, k, R, H, n, _ptr(dx), _ptr(dweights), _stream_on(stream, dev))
    if status:
        _check(status)
    return dx, dweights


def _dots(other, what, shape, dtype, dweights, dshape, device, stream):
    """The weights' gradients, where the other factor of their products is given."""
    if other is None:
        if dweights is not None:
            raise ValueError(f"dweights needs {what}")
        return None
    _operand(other, what, dtype, shape, device)
    return _out(dweights, dshape, _F32, device, "dweights", stream)


def pcm_combine_rows(o: torch.Tensor, row_of: torch.Tensor, weights=None, offsets=None, y=None,
                     out_dtype: Optional[torch.dtype] = None, accumulate: bool = False, stream=None) -> torch.Tensor:
    """y[t] = [y[t] +] the sum of weights[t, a] o[row_of[t, a]] over the slots. accumulate adds into y, which is then
    float32. row_of outside the groups' rows: none."""
    R, H = _matrix(o, "o")
    _operand(o, "o")
    dev = o.device
    T, k, n = _slots(row_of, weights, offsets, dev)
    if accumulate and y is None:
        raise ValueError("accumulate needs y")
    out = _out_type(y, out_dtype, o.dtype)
    y = _out(y, (T, H), out, dev, "y", stream)
    status = lib().pcm_combine_rows(_code(o.dtype), _code(out), _ptr(o), _ptr(row_of), _ptr(weights), _ptr(offsets), T, k, R, H, n,
                                    _ptr(y), int(bool(accumulate)), _stream_on(stream, dev))
    if status:
        _check(status)
    return y


def pcm_combine_rows_grad(dy: torch.Tensor, row_of: torch.Tensor, o: Optional[torch.Tensor] = None, weights=None, offsets=None,
                          rows: Optional[int] = None, do=None, dweights=None, out_dtype: Optional[torch.dtype] = None,
                          stream=None):
    """(do, dweights) of pcm_combine_rows: do[row_of[t, a]] = weights[t, a] dy[t], and, with o, the products
    <o[row_of[t, a]], dy[t]> (None without). do has o's rows (or `rows`, T k by default); rows of no pair are left as
    they were (in a `do` that the caller does not pass: undefined). o may be of the other type."""
    T, H = _matrix(dy, "dy")
    _operand(dy, "dy")
    dev = dy.device
    t, k, n = _slots(row_of, weights, offsets, dev)
    if t != T:
        raise ValueError("row_of must have a row for each token")
    if o is not None:
        rows = _row_count(rows, o, T, k)
    R = _row_count(rows, do, T, k)
    out = _out_type(do, out_dtype, dy.dtype)
    dweights = _dots(o, "o", (R, H), None, dweights, (T, k), dev, stream)
    do = _out(do, (R, H), out, dev, "do", stream)
    status = lib().pcm_combine_rows_grad(_code(dy.dtype), _code((dy if o is None else o).dtype), _code(out), _ptr(dy), _ptr(o), _ptr(row_of), _ptr(weights),
                                         _ptr(offsets), T, k, R, H, n, _ptr(do), _ptr(dweights), _stream_on(stream, dev))
    if status:
        _check(status)
    return do, dweights


def _halves(gate_up):
    if gate_up.dim() != 2 or gate_up.shape[1] % 2:
        raise ValueError("gate_up must have two dimensions and an even number of columns")
    R, F = gate_up.shape[0], gate_up.shape[1] // 2
    if F > _INT_MAX:
        _too_wide("gate_up")
    _operand(gate_up, "gate_up")
    return R, F


def pcm_swiglu(gate_up: torch.Tensor, count=None, u=None, out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """SiLU(gate) * up; gate_up [R, 2F] holds a row's gate values before its up values. count: one int32 on the device (such
    as offsets[-1]); rows from there on are left as they were."""
    R, F = _halves(gate_up)
    dev = gate_up.device
    _count(count, dev)
    out = _out_type(u, out_dtype, gate_up.dtype)
    u = _out(u, (R, F), out, dev, "u", stream)
    status = lib().pcm_swiglu(_code(gate_up.dtype), _code(out), _ptr(gate_up), _ptr(count), R, F, _ptr(u), _stream_on(stream, dev))
    if status:
        _check(status)
    return u


def pcm_swiglu_grad(gate_up: torch.Tensor, du: torch.Tensor, count=None, dgate_up=None, out_dtype: Optional[torch.dtype] = None,
                    stream=None) -> torch.Tensor:
    """The gradient of pcm_swiglu by gate_up, [R, 2F], from gate_up and du [R, F]."""
    R, F = _halves(gate_up)
    dev = gate_up.device
    _operand(du, "du", gate_up.dtype, (R, F), dev)
    _count(count, dev)
    out = _out_type(dgate_up, out_dtype, gate_up.dtype)
    dgate_up = _out(dgate_up, (R, 2 * F), out, dev, "dgate_up", stream)
    status = lib().pcm_swiglu_grad(_code(gate_up.dtype), _code(out), _ptr(gate_up), _ptr(du), _ptr(count), R, F, _ptr(dgate_up),
                                   _stream_on(stream, dev))
    if status:
        _check(status)
    return dgate_up


def _path_table(path_bits, beta, src_row_of, tgt_row_of, device):
    T, k = _table(src_row_of, "src_row_of", device)
    if tgt_row_of is None:
        tgt_row_of = src_row_of
    else:
        _table(tgt_row_of, "tgt_row_of", device, (T, k))
    _operand(path_bits, "path_bits", torch.int64, (T,), device)
    _operand(beta, "beta", _F32, (T, k, k), device)
    return T, k, tgt_row_of


def pcm_mix_rows(u: torch.Tensor, path_bits: torch.Tensor, beta: torch.Tensor, src_row_of: torch.Tensor, tgt_row_of=None,
                 rows: Optional[int] = None, z=None, out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """z[tgt_row_of[t, b]] = the sum of beta[t, a, b] u[src_row_of[t, a]] over the paths (a, b) of token t. tgt_row_of:
    src_row_of by default. z has `rows` rows (u's by default); rows of no pair are left as they were."""
    R, F = _matrix(u, "u")
    _operand(u, "u")
    dev = u.device
    T, k, tgt_row_of = _path_table(path_bits, beta, src_row_of, tgt_row_of, dev)
    out = _out_type(z, out_dtype, u.dtype)
    R_tgt = R if rows is None and z is None else _row_count(rows, z, T, k)
    z = _out(z, (R_tgt, F), out, dev, "z", stream)
    status = lib().pcm_mix_rows(_code(u.dtype), _code(out), _ptr(u), _ptr(path_bits), _ptr(beta), _ptr(src_row_of),
                                _ptr(tgt_row_of), T, k, R, R_tgt, F, _ptr(z), _stream_on(stream, dev))
    if status:
        _check(status)
    return z


def pcm_mix_rows_grad(dz: torch.Tensor, u: Optional[torch.Tensor], path_bits: torch.Tensor, beta: torch.Tensor,
                      src_row_of: torch.Tensor, tgt_row_of=None, rows: Optional[int] = None, du=None, dbeta=None,
                      out_dtype: Optional[torch.dtype] = None, stream=None):
    """(du, dbeta) of pcm_mix_rows: du[src_row_of[t, a]] = the sum of beta[t, a, b] dz[tgt_row_of[t, b]] over the paths, and
    dbeta[t, a, b] = <dz[tgt_row_of[t, b]], u[src_row_of[t, a]]>, 0 where there is no path (None where u is None). du has
    u's rows (or `rows`, dz's by default)."""
    R, F = _matrix(dz, "dz")
    _operand(dz, "dz")
    dev = dz.device
    T, k, tgt_row_of = _path_table(path_bits, beta, src_row_of, tgt_row_of, dev)
    if u is not None:
        rows = _row_count(rows, u, T, k)
    R_src = R if rows is None and du is None else _row_count(rows, du, T, k)
    out = _out_type(du, out_dtype, dz.dtype)
    dbeta = _dots(u, "u", (R_src, F), dz.dtype, dbeta, (T, k, k), dev, stream)
    du = _out(du, (R_src, F), out, dev, "du", stream)
    status = lib().pcm_mix_rows_grad(_code(dz.dtype), _code(out), _ptr(dz), _ptr(u), _ptr(path_bits), _ptr(beta),
                                     _ptr(src_row_of), _ptr(tgt_row_of), T, k, R_src, R, F, _ptr(du), _ptr(dbeta),
                                     _stream_on(stream, dev))
    if status:
        _check(status)
    return du, dbeta


def pcm_route_grad(topk_ids: torch.Tensor, topk_w: torch.Tensor, n: int, path_bits=None, dbeta=None, dw=None,
                   beta_mode: int = BETA_SRC_COND, dlogits=None, out_dtype: Optional[torch.dtype] = None,
                   stream=None) -> torch.Tensor:
    """dlogits [T, n] (float32 by default) from dbeta [T, k, k] by the path weights (of the paths in path_bits, under
    beta_mode) and dw [T, k] by topk_w, either or both. 0 for the logits that were not selected."""
    T, k = _matrix(topk_ids, "topk_ids")
    _operand(topk_ids, "topk_ids", torch.int32)
    dev = topk_ids.device
    _operand(topk_w, "topk_w", _F32, (T, k), dev)
    if (path_bits is None) != (dbeta is None):
        raise ValueError("path_bits and dbeta come together")
    if dbeta is not None:
        _operand(path_bits, "path_bits", torch.int64, (T,), dev)
        _operand(dbeta, "dbeta", _F32, (T, k, k), dev)
    if dw is not None:
        _operand(dw, "dw", _F32, (T, k), dev)
    if n > _INT_MAX:
        _too_wide("n")
    out = _out_type(dlogits, out_dtype, _F32)
    dlogits = _out(dlogits, (T, n), out, dev, "dlogits", stream)
    status = lib().pcm_route_grad(_code(out), _ptr(topk_ids), _ptr(topk_w), _ptr(path_bits), _ptr(dbeta), beta_mode, _ptr(dw), T, n,
                                  k, _ptr(dlogits), _stream_on(stream, dev))
    if status:
        _check(status)
    return dlogits


# ------------------------------------------------------------------------ all gradients
def _tensors(tensors: Sequence[torch.Tensor], what: str):
    """The pcm_tensor array of the tensors (three 64-bit words each), and their counts. (The five attributes cost 30 to 55 ns
    each, 0.22 us a tensor: taken by maps, packed by slices.)"""
    T = torch.Tensor
    devices = set(map(T.get_device, tensors))
    if devices and (min(devices) < 0 or devices != {torch.cuda.current_device()} or not all(map(T.is_contiguous, tensors))):
        raise ValueError(f"{what} must be contiguous tensors on the current device")
    try:
        codes = [_CODES[t.dtype] for t in tensors]
    except KeyError as e:
        raise TypeError(f"unsupported dtype {e.args[0]}: float32 or bfloat16") from None
    counts = array("Q", map(T.numel, tensors))
    words = array("Q", bytes(24 * len(codes)))
    words[0::3], words[1::3], words[2::3] = array("Q", map(T.data_ptr, tensors)), counts, array("Q", codes)
    return words, counts


def _address(words: Optional[array]):
    return words.buffer_info()[0] if words else None


def _listed(tensors):
    """What can be read more than once: an iterator would come back empty."""
    return tensors if isinstance(tensors, (list, tuple)) else list(tensors)


def _clipped(grads, out):
    """The arrays of grads and of out (None in place), and their device."""
    words, counts = _tensors(grads, "grads")
    to = None
    if out is not None:
        to, others = _tensors(out, "out")
        if others != counts:
            raise ValueError("out must have as many elements as grads, tensor by tensor")
    return words, to, _device(grads)


def _device(tensors):
    return tensors[0].device if tensors else torch.device("cuda", torch.cuda.current_device())


def _one(norm, device):
    if norm.numel() != 1:
        raise ValueError("norm must be one number")
    _operand(norm, "norm", _F32, None, device)
    return norm


def _norm_out(norm, device, stream):
    return _out(None, (1,), _F32, device, "norm", stream) if norm is None else _one(norm, device)


def pcm_grad_norm(grads: Sequence[torch.Tensor], norm=None, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The norm over every element of all gradients, [1] float32 on the device; squares and sums in 64 bits.
    ws: workspace_bytes(OP_GRAD_NORM, len(grads), 0, 0, 1, 1, 0) bytes."""
    grads = list(grads)
    words, _ = _tensors(grads, "grads")
    dev = _device(grads)
    norm = _norm_out(norm, dev, stream)
    ws = _workspace(ws, workspace_bytes(OP_GRAD_NORM, len(grads), 0, 0, 1, 1, 0), dev, stream)
    status = lib().pcm_grad_norm(_address(words), len(grads), _ptr(norm), _ptr(ws), ws.numel(), _stream_on(stream, dev))
    if status:
        _check(status)
    return norm


def pcm_clip_grads(grads: Sequence[torch.Tensor], norm: torch.Tensor, max_norm: float, out=None, stream=None):
    """Where norm (one float32 on the device) is over max_norm, the gradients times max_norm / norm; as they are where it is
    not, or is not finite. In place, or into the tensors of `out` (of either type). Gradients must not overlap. Returns
    out, or grads: the list or tuple itself, of another iterable a list."""
    if norm is None:
        raise ValueError("norm must be given: pcm_clip_grad_norm forms it")
    grads, out = _listed(grads), None if out is None else _listed(out)
    words, to, dev = _clipped(grads, out)
    _one(norm, dev)
    status = lib().pcm_clip_grads(_address(words), _address(to), len(grads), _ptr(norm), float(max_norm),
                                  _stream_on(stream, dev))
    if status:
        _check(status)
    return grads if out is None else out


def pcm_clip_grad_norm(grads: Sequence[torch.Tensor], max_norm: float, out=None, norm=None, ws: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """pcm_grad_norm and pcm_clip_grads with that norm, the same results; returns the norm."""
    grads = list(grads)
    words, to, dev = _clipped(grads, None if out is None else list(out))
    norm = _norm_out(norm, dev, stream)
    ws = _workspace(ws, workspace_bytes(OP_GRAD_NORM, len(grads), 0, 0, 1, 1, 0), dev, stream)
    status = lib().pcm_clip_grad_norm(_address(words), _address(to), len(grads), float(max_norm), _ptr(norm),
                                      _ptr(ws), ws.numel(), _stream_on(stream, dev))
    if status:
        _check(status)
    return norm
