"""The attention sublayer of present-day blocks, operator by operator, on torch tensors: norms of queries and keys with the position rotation, attention with a
learned relative position bias, dropout with the residual sum, and their gradients.

Argument marshalling only: shapes, types and strides are checked here and in the library, results and workspaces are torch's memory, and every call goes to the current
stream of the tensors' device.  Tensors are CUDA tensors whose last dimension is contiguous; other strides are free (zgr.h says in which units).
"""
import ctypes as C
from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.float32: B.ZGR_F32, torch.bfloat16: B.ZGR_BF16}
_U64 = (1 << 64) - 1


def _dtype(t, name):
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise TypeError(f"{name} is {t.dtype}: float32 or bfloat16 is wanted") from None


def _want(ok, what):
    if not ok:
        raise ValueError(what)


def _vector(t, n, dtype, device, name):
    """The address of a contiguous vector (or table) of n entries, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise TypeError(f"{name} is {t.dtype}: {dtype} is wanted")
    _want(t.numel() == n and t.is_contiguous() and t.device == device, f"{name}: {n} contiguous entries on {device} are wanted")
    return t.data_ptr()


def _view(t, name, like=None):
    """zgr_heads of a [batch, tokens, heads, dim] or [tokens, heads, dim] tensor."""
    _want(t.is_cuda, f"{name} must be on the GPU")
    if like is not None:
        _want(t.shape == like.shape and t.dtype is like.dtype and t.device == like.device, f"{name} must have the shape, type and device of what it belongs to")
    s = t.stride()
    _want(s[-1] == 1 or t.shape[-1] == 1, f"{name}: the last dimension must be contiguous")
    return B.zgr_heads(t.data_ptr(), s[0] if t.dim() == 4 else 0, s[-3], s[-2])


class _On:
    """The device and its current stream: a launch goes to the device that is current."""
    __slots__ = ("device", "guard")

    def __init__(self, device):
        self.device = device
        self.guard = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


# ---- norms of queries and keys, with the position rotation ----------------------------------------------------
def rotation_table(n_positions, rot_dim, base=10000.0, device="cuda:0"):
    """fp32 [n_positions, rot_dim / 2, 2]: cosine and sine of position base^(-2 i / rot_dim), taken in 64 bits."""
    angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * float(base) ** (-2.0 * torch.arange(rot_dim // 2, dtype=torch.float64) / rot_dim)
    return torch.stack([angle.cos(), angle.sin()], -1).to(torch.float32).to(device)


def _rotation(q, k, q_gain, k_gain, table, positions, eps, interleaved):
    x = q if q is not None else k
    _want(x is not None, "q or k is wanted")
    _want(x.dim() == 3 and (q is None or k is None or (k.dim() == 3 and k.shape[0] == q.shape[0] and k.shape[2] == q.shape[2] and k.dtype is q.dtype and k.device == q.device)),
          "q and k: [tokens, heads, dim] of one type on one device")
    rows, _, dim = x.shape
    rot = 0 if table is None else 2 * table.shape[1]
    if table is not None:
        _want(table.dim() == 3 and table.shape[2] == 2, "table: [positions, rot_dim / 2, 2]")
    return B.zgr_rotation(_dtype(x, "q"), rows, 0 if q is None else q.shape[1], 0 if k is None else k.shape[1], dim, rot, 1 if interleaved else 0, 0 if table is None else table.shape[0], eps,
                          _vector(q_gain, dim, x.dtype, x.device, "q_gain"), _vector(k_gain, dim, x.dtype, x.device, "k_gain"),
                          None if table is None else _vector(table, table.numel(), torch.float32, x.device, "table"),
                          None if table is None else _vector(positions, rows, torch.int32, x.device, "positions")), x


def _ref(view):
    return None if view is None else C.byref(view)


def norm_rotate(q, k, q_gain, k_gain, table, positions, eps=1e-6, interleaved=False, q_out=None, k_out=None):
    """(q, k) normalised for each head and rotated: q [tokens, heads, dim], k [tokens, k_heads, dim] (one may be None), gains [dim] or None (not normalised), table
    as rotation_table makes it or None (no rotation), positions int32 [tokens].  q_out, k_out: where the results go (q and k themselves are allowed)."""
    how, x = _rotation(q, k, q_gain, k_gain, table, positions, eps, interleaved)
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is not None and k_out is None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    views = [None if t is None else _view(t, n, like) for t, n, like in ((q, "q", None), (k, "k", None), (q_out, "q_out", q), (k_out, "k_out", k))]
    with _On(x.device) as stream:
        B.check(B.lib().zgr_norm_rotate(C.byref(how), *map(_ref, views), stream))
    return q_out, k_out


def norm_rotate_backward(dq_out, dk_out, q, k, q_gain, k_gain, table, positions, eps=1e-6, interleaved=False):
    """(dq, dk, dq_gain, dk_gain) from the gradients of norm_rotate's results and its inputs; the gains' gradients are fp32, None where there is no gain."""
    how, x = _rotation(q, k, q_gain, k_gain, table, positions, eps, interleaved)
    dq, dk = (None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
    views = [None if t is None else _view(t, n, like) for t, n, like in ((dq_out, "dq_out", q), (dk_out, "dk_out", k), (q, "q", None), (k, "k", None), (dq, "dq", None), (dk, "dk", None))]
    lib = B.lib()
    gains = ws = None
    n = 0
    if q_gain is not None or k_gain is not None:
        n = lib.zgr_norm_rotate_backward_workspace(C.byref(how))
        gains = torch.empty(2, x.shape[2], dtype=torch.float32, device=x.device)
        ws = torch.empty(n, dtype=torch.uint8, device=x.device)
    with _On(x.device) as stream:
        B.check(lib.zgr_norm_rotate_backward(C.byref(how), *map(_ref, views), None if gains is None else gains.data_ptr(), None if ws is None else ws.data_ptr(), n, stream))
    return dq, dk, None if q_gain is None else gains[0], None if k_gain is None else gains[1]


# ---- attention with a relative position bias ------------------------------------------------------------------
def relative_buckets(buckets, reach, causal, device="cuda:0"):
    """int32 [2 reach + 1]: the bucket of each relative position key - query in [-reach, reach] (zgr_relative_buckets)."""
    out = (C.c_int32 * (2 * reach + 1))()
    B.check(B.lib().zgr_relative_buckets(buckets, reach, 1 if causal else 0, out))
    return torch.tensor(list(out), dtype=torch.int32, device=device)


def _attention(q, k, v, bias, bias_map, causal, scale, q_lengths, k_lengths, q_start):
    _want(q.dim() == 4 and k.dim() == 4 and k.shape == v.shape and k.shape[0] == q.shape[0] and k.shape[3] == q.shape[3], "q: [batch, tokens, heads, dim], k and v: [batch, keys, kv_heads, dim]")
    _want(k.dtype is q.dtype and v.dtype is q.dtype and k.device == q.device and v.device == q.device, "q, k and v must have one type and device")
    b, n_q, heads, dim = q.shape
    reach = buckets = 0
    if bias is not None:
        _want(bias.dim() == 2 and bias.shape[1] == heads and bias_map is not None and bias_map.numel() % 2 == 1, "bias: [buckets, heads], bias_map: [2 reach + 1]")
        buckets, reach = bias.shape[0], bias_map.numel() // 2
    dev = q.device
    return B.zgr_attention(_dtype(q, "q"), b, n_q, k.shape[1], heads, k.shape[2], dim, 1 if causal else 0, dim ** -0.5 if scale is None else scale,
                           _vector(q_lengths, b, torch.int32, dev, "q_lengths"), _vector(k_lengths, b, torch.int32, dev, "k_lengths"), _vector(q_start, b, torch.int32, dev, "q_start"),
                           None if bias is None else _vector(bias, buckets * heads, q.dtype, dev, "bias"), None if bias is None else _vector(bias_map, 2 * reach + 1, torch.int32, dev, "bias_map"),
                           buckets, reach)


def attention(q, k, v, bias=None, bias_map=None, causal=False, scale: Optional[float] = None, q_lengths=None, k_lengths=None, q_start=None, out=None):
    """(out, lse) of zgr_attention_forward: q [batch, n_q, heads, dim], k and v [batch, n_k, kv_heads, dim], bias [buckets, heads] with bias_map int32 [2 reach + 1] (relative_buckets),
    lengths and starts int32 [batch]; scale: 1 / sqrt(dim) unless given.  lse: fp32 [batch, heads, n_q]."""
    how = _attention(q, k, v, bias, bias_map, causal, scale, q_lengths, k_lengths, q_start)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[0], q.shape[2], q.shape[1], dtype=torch.float32, device=q.device)
    views = (_view(q, "q"), _view(k, "k"), _view(v, "v"), _view(out, "out", q))
    lib = B.lib()
    n = lib.zgr_attention_workspace(C.byref(how))
    ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    with _On(q.device) as stream:
        B.check(lib.zgr_attention_forward(C.byref(how), *map(C.byref, views), lse.data_ptr(), None if ws is None else ws.data_ptr(), n, stream))
    return out, lse


def attention_backward(dout, q, k, v, out, lse, bias=None, bias_map=None, causal=False, scale: Optional[float] = None, q_lengths=None, k_lengths=None, q_start=None):
    """(dq, dk, dv, dbias) from the gradient of attention's `out`, its inputs and its results; dbias is None without a bias."""
    how = _attention(q, k, v, bias, bias_map, causal, scale, q_lengths, k_lengths, q_start)
    _want(lse.dtype is torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (q.shape[0], q.shape[2], q.shape[1]) and lse.device == q.device, "lse: what attention returned")
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
    dbias = None if bias is None else torch.empty(bias.shape, dtype=bias.dtype, device=bias.device)
    views = (_view(dout, "dout", q), _view(q, "q"), _view(k, "k"), _view(v, "v"), _view(out, "out", q))
    grads = (_view(dq, "dq"), _view(dk, "dk"), _view(dv, "dv"))
    lib = B.lib()
    n = lib.zgr_attention_backward_workspace(C.byref(how))
    ws = torch.empty(n, dtype=torch.uint8, device=q.device)
    with _On(q.device) as stream:
        B.check(lib.zgr_attention_backward(C.byref(how), *map(C.byref, views), lse.data_ptr(), *map(C.byref, grads), None if dbias is None else dbias.data_ptr(), ws.data_ptr(), n, stream))
    return dq, dk, dv, dbias


# ---- dropout with the residual sum ----------------------------------------------------------------------------
def _rows(t, name):
    _want(t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1), f"{name}: [rows, cols] on the GPU with contiguous rows")
    return t.data_ptr()


def dropout_add(x, bias, residual, p, seed, step, site, first_row=0, out=None):
    """residual + dropout(x + bias) [rows, cols]: zgr_dropout_add.  bias [cols] in x's type or None; residual and the result share a type (x's where residual is None)."""
    rows, cols = x.shape
    stream_type = x.dtype if residual is None else residual.dtype
    if out is None:
        out = torch.empty(rows, cols, dtype=stream_type, device=x.device)
    for t, n in ((residual, "residual"), (out, "out")):
        _want(t is None or (t.shape == x.shape and t.dtype is stream_type and t.device == x.device), f"{n} must have x's shape and device and the residual's type")
    with _On(x.device) as stream:
        B.check(B.lib().zgr_dropout_add(rows, cols, _dtype(x, "x"), _rows(x, "x"), x.stride(0), _vector(bias, cols, x.dtype, x.device, "bias"), _dtype(out, "residual"),
                                        None if residual is None else _rows(residual, "residual"), 0 if residual is None else residual.stride(0), _rows(out, "out"), out.stride(0),
                                        p, seed & _U64, step, site, first_row, stream))
    return out


def dropout_add_backward(dout, x_dtype, p, seed, step, site, first_row=0, want_bias=True):
    """(dx, dbias) from the gradient of dropout_add's result: dx in x_dtype, dbias fp32 [cols] or None.  The residual's gradient is dout itself."""
    rows, cols = dout.shape
    dx = torch.empty(rows, cols, dtype=x_dtype, device=dout.device)
    dbias = ws = None
    n = 0
    lib = B.lib()
    if want_bias:
        n = lib.zgr_dropout_add_backward_workspace(rows, cols)
        dbias = torch.empty(cols, dtype=torch.float32, device=dout.device)
        ws = torch.empty(n, dtype=torch.uint8, device=dout.device)
    with _On(dout.device) as stream:
        B.check(lib.zgr_dropout_add_backward(rows, cols, _dtype(dout, "dout"), _rows(dout, "dout"), dout.stride(0), _dtype(dx, "dx"), dx.data_ptr(), cols,
                                             None if dbias is None else dbias.data_ptr(), p, seed & _U64, step, site, first_row, None if ws is None else ws.data_ptr(), n, stream))
    return dx, dbias
