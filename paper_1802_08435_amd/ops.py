"""Operators on GPU tensors that need no model (``include/wavernn.h``): log
probabilities of given tokens with entropy and top alternatives, table lookup,
layer norm, and the gradient of each.

Argument marshalling only, as in ``wavernn``.  Rows are the last dimension, whose
elements are adjacent; the dimensions before it may be any view with one distance
between rows (a slice of wider rows, an expanded row).  Tensors of one call are on
one GPU, which need not be the current one; the call runs on ``stream`` (default:
that GPU's current stream), and tensors it allocates belong to that stream.  Wrong
shapes, types or devices raise ``ValueError`` before anything is launched.  No
function takes part in torch's autograd: a gradient is a call of its own.
"""
from __future__ import annotations

import torch

from . import wavernn as _w

MAX_TOP = 32
# (torch.cuda.current_stream() makes an object, which takes 2.6 us of a small call's 9; a torch without GPU
# support has neither, and no tensor that gets as far as them)
_raw_stream, _current_gpu = (getattr(torch._C, k, None) for k in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
_DTYPE = {torch.float32: _w.F32, torch.bfloat16: _w.BF16, torch.float16: _w.F16}
_ID_BYTES = {torch.int32: 4, torch.int64: 8}


def _dtype(name, t):
    if t.dtype not in _DTYPE:
        raise ValueError(f"{name}: dtype {t.dtype} is not float32, bfloat16 or float16")
    return _DTYPE[t.dtype]


def _rows(name, t):
    """(rows, elements of a row, elements from row to row) of t [..., width]."""
    shape = t.shape
    if len(shape) == 2:
        n, w = shape
        step, one = t.stride()
        if one != 1 and w > 1:
            raise ValueError(f"{name}: the elements of a row must be adjacent")
        return n, w, step if n > 1 else w
    if not shape:
        raise ValueError(f"{name}: needs a last dimension of elements")
    w = shape[-1]
    if w > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    if t.dim() == 1:
        return 1, w, w
    n = 1
    for s in t.shape[:-1]:
        n *= s
    if n == 0 or t.is_contiguous():
        return n, w, w
    step, run = None, 1                    # from the last leading dimension outwards
    for d in range(t.dim() - 2, -1, -1):
        if t.shape[d] == 1:
            continue
        if step is None:
            step = t.stride(d)
        elif t.stride(d) != step * run:
            raise ValueError(f"{name}: the rows are not one distance apart (take a contiguous copy, or the whole rows with padding)")
        run *= t.shape[d]
    return n, w, w if step is None else step


def _plain(name, t, shape, dtypes, device):
    """t's address (None for None), t checked to be contiguous, of the shape, on the device and of one of the dtypes."""
    if t is None:
        return None
    if t.shape == shape and t.dtype in dtypes and t.device == device and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: needs a contiguous tensor {list(shape)} on {device}, {' or '.join(str(d) for d in dtypes)}; "
                     f"got {t.dtype} {list(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")


def _result(name, out, shape, dtype, like):
    """A new tensor, or ``out`` checked to fit; with the distance between its rows."""
    if out is None:
        return like.new_empty(shape, dtype=dtype), shape[-1]
    device = like.device
    if out.shape != shape or out.dtype != dtype or out.device != device:
        raise ValueError(f"{name}: needs {dtype} {list(shape)} on {device}, got {out.dtype} {list(out.shape)} on {out.device}")
    return out, _rows(name, out)[2]


def _workspace(n_bytes, like):
    return like.new_empty(n_bytes, dtype=torch.uint8) if n_bytes > 0 else None


def _p(t):
    return None if t is None else t.data_ptr()


def _away(t, stream):
    """Is a call on t for another stream or GPU than the current ones?"""
    gpu = t.device.index
    return stream is not None or gpu is None or gpu != _current_gpu()


def _there(fn, t, stream, *args):
    """fn(*args) with t's GPU current and, if a stream is given, that stream."""
    if not t.is_cuda:
        raise ValueError(f"{fn.__name__}: tensors must be on a GPU")
    if stream is not None and stream.device != t.device:
        raise ValueError(f"{fn.__name__}: the stream is on {stream.device}, the tensors on {t.device}")
    with torch.cuda.device(t.device), torch.cuda.stream(stream):
        return fn(*args)


_F32 = (torch.float32,)
_I32 = (torch.int32,)
_IDS = (torch.int64, torch.int32)


def token_logprobs(logits, tokens=None, top=0, stream=None):
    """Log probability of tokens [...] under logits [..., V], with the entropy, the log of the
    sum and the ``top`` most likely classes of every distribution: a dict of logp (None
    without tokens), entropy, lse [...], top_logp and top_idx [..., top] (None with top = 0), fp32 and
    int32.  tokens are int64 or int32; a negative one marks a row of padding, which is
    not read and gives 0 (top_idx -1).  Masked classes are -inf.  Tokens one place ahead of their logits [B, T, V]
    need no copy: give all T rows, with the tokens shifted and -1 in the last place (logits[:, :-1] is
    refused, its rows being two distances apart).  Edge cases and the order of
    alternatives: include/wavernn.h, wavernn_token_logprobs."""
    if _away(logits, stream):
        return _there(token_logprobs, logits, stream, logits, tokens, top)
    L = _w._lib or _w.lib()
    dt, (n, v, stride), dev, shape = _dtype("logits", logits), _rows("logits", logits), logits.device, logits.shape[:-1]
    tokens_p = _plain("tokens", tokens, shape, _IDS, dev)
    ws_bytes = L.wavernn_token_logprobs_workspace(n, v, top)
    ws = _workspace(ws_bytes, logits)
    logp = None
    if tokens is not None:                 # one allocation for the three
        logp, entropy, lse = logits.new_empty((3, *shape), dtype=torch.float32).unbind()
    else:
        entropy, lse = logits.new_empty((2, *shape), dtype=torch.float32).unbind()
    top_logp = top_idx = None
    if top > 0:
        top_logp = logits.new_empty((*shape, top), dtype=torch.float32)
        top_idx = logits.new_empty((*shape, top), dtype=torch.int32)
    _w._check(L.wavernn_token_logprobs(dt, logits.data_ptr(), n, v, stride, tokens_p,
                                       0 if tokens is None else _ID_BYTES[tokens.dtype], top, _p(logp),
                                       entropy.data_ptr(), lse.data_ptr(), _p(top_logp), _p(top_idx), _p(ws),
                                       max(ws_bytes, 0), _raw_stream(dev.index)))
    return dict(logp=logp, entropy=entropy, lse=lse, top_logp=top_logp, top_idx=top_idx)


def token_logprobs_grad(logits, tokens, lse, entropy=None, g_logp=None, g_entropy=None, g_lse=None, top_idx=None,
                        g_top=None, out=None, stream=None):
    """Gradient with respect to the logits of a loss whose gradients with respect to
    token_logprobs' results are g_logp, g_entropy, g_lse [...] and g_top [..., top] (of top_logp; any
    may be None), given the results lse, entropy (for g_entropy) and top_idx (for g_top).  The
    probabilities are exp(logits - lse), as good as lse's fp32 rounding.
    ``out`` may be the logits themselves."""
    if _away(logits, stream):
        return _there(token_logprobs_grad, logits, stream, logits, tokens, lse, entropy, g_logp, g_entropy, g_lse, top_idx,
                      g_top, out)
    L = _w._lib or _w.lib()
    dt, (n, v, stride), dev, shape = _dtype("logits", logits), _rows("logits", logits), logits.device, logits.shape[:-1]
    tokens_p = _plain("tokens", tokens, shape, _IDS, dev)
    k, top_p, g_top_p = 0, None, None
    if g_top is not None:
        k = g_top.shape[-1] if g_top.dim() else -1
        g_top_p = _plain("g_top", g_top, shape + (k,), _F32, dev)
        if top_idx is None:
            raise ValueError("g_top needs top_idx")
        top_p = _plain("top_idx", top_idx, shape + (k,), _I32, dev)
    out, out_stride = _result("out", out, logits.shape, logits.dtype, logits)
    _w._check(L.wavernn_token_logprobs_grad(dt, logits.data_ptr(), n, v, stride, tokens_p,
                                            0 if tokens is None else _ID_BYTES[tokens.dtype],
                                            _plain("lse", lse, shape, _F32, dev), _plain("entropy", entropy, shape, _F32, dev),
                                            _plain("g_logp", g_logp, shape, _F32, dev),
                                            _plain("g_entropy", g_entropy, shape, _F32, dev),
                                            _plain("g_lse", g_lse, shape, _F32, dev), k, top_p, g_top_p, out.data_ptr(),
                                            out_stride, _raw_stream(dev.index)))
    return out


def _table_dtype(name, dtype, like):
    dtype = like if dtype is None else dtype
    if dtype != like and dtype != torch.float32:
        raise ValueError(f"{name}: dtype must be {like} or float32")
    return dtype


def embed(table, ids, scale=1.0, dtype=None, out=None, stream=None):
    """scale * table[ids]: rows of table [V, d] for ids [...] (int64 or int32) as [..., d], of the
    table's dtype or float32.  A negative id is padding (zeros); one of V or more gives NaN.
    ``out`` [..., d] may be a slice of wider rows."""
    if _away(table, stream):
        return _there(embed, table, stream, table, ids, scale, dtype, out)
    L = _w._lib or _w.lib()
    dt, dev = _dtype("table", table), table.device
    if table.dim() != 2:
        raise ValueError("table: needs two dimensions")
    v, d, stride = _rows("table", table)
    ids_p = _plain("ids", ids, ids.shape, _IDS, dev)
    dtype = _table_dtype("embed", dtype, table.dtype)
    out, out_stride = _result("out", out, ids.shape + (d,), dtype, table)
    _w._check(L.wavernn_embed(dt, table.data_ptr(), v, d, stride, ids_p, _ID_BYTES[ids.dtype], ids.numel(), scale,
                              _DTYPE[dtype], out.data_ptr(), out_stride, _raw_stream(dev.index)))
    return out


def embed_grad(dout, ids, n_rows, scale=1.0, dtype=torch.float32, stream=None):
    """Gradient of embed's table [n_rows, d] from dout [..., d] and ids [...]: scale times
    the sum of dout's rows for each number, zero for numbers that do not occur; sums in fp32 in an
    order of their own, the same every time.  dtype: float32 or dout's."""
    if _away(dout, stream):
        return _there(embed_grad, dout, stream, dout, ids, n_rows, scale, dtype)
    L = _w._lib or _w.lib()
    dt, (n, d, stride), dev = _dtype("dout", dout), _rows("dout", dout), dout.device
    ids_p = _plain("ids", ids, dout.shape[:-1], _IDS, dev)
    dtype = _table_dtype("embed_grad", dtype, dout.dtype)
    ws_bytes = L.wavernn_embed_grad_workspace(n, d, n_rows)
    ws = _workspace(ws_bytes, dout)
    out = dout.new_empty((max(n_rows, 0), d), dtype=dtype)
    _w._check(L.wavernn_embed_grad(dt, dout.data_ptr(), n, d, stride, ids_p, _ID_BYTES[ids.dtype], n_rows, scale,
                                   _DTYPE[dtype], out.data_ptr(), _p(ws), max(ws_bytes, 0), _raw_stream(dev.index)))
    return out


def _weight(name, w, d, t, other=None):
    if w is None:
        return None
    if other is not None and w.dtype != other.dtype:
        raise ValueError("gamma and beta must be of one dtype")
    return _plain(name, w, (d,), (torch.float32, t.dtype), t.device)


def layer_norm(x, gamma=None, beta=None, eps=1e-5, stats=False, out=None, stream=None):
    """(x - mean) / sqrt(variance + eps) * gamma + beta over the last dimension of x [..., d], of x's
    dtype; gamma, beta [d] of x's dtype or float32.  With ``stats`` also the rows' mean and
    1 / sqrt(variance + eps) [...], which layer_norm_grad takes.  ``out`` may be x."""
    if _away(x, stream):
        return _there(layer_norm, x, stream, x, gamma, beta, eps, stats, out)
    L = _w._lib or _w.lib()
    dt, (n, d, stride), dev = _dtype("x", x), _rows("x", x), x.device
    gamma_p = _weight("gamma", gamma, d, x)
    beta_p = _weight("beta", beta, d, x, gamma)
    w = gamma if gamma is not None else beta
    y, y_stride = _result("out", out, x.shape, x.dtype, x)
    mean = rstd = None
    if stats:
        mean, rstd = x.new_empty((2, *x.shape[:-1]), dtype=torch.float32).unbind()
    _w._check(L.wavernn_layer_norm(dt, x.data_ptr(), n, d, stride, _w.F32 if w is None else _DTYPE[w.dtype], gamma_p,
                                   beta_p, eps, y.data_ptr(), y_stride, _p(mean), _p(rstd), _raw_stream(dev.index)))
    return (y, mean, rstd) if stats else y


def layer_norm_grad(dy, x, mean, rstd, gamma=None, weights=True, out=None, stream=None):
    """(dx, dgamma, dbeta) of layer_norm from dy [..., d], its x and the statistics it
    returned; dx of x's dtype, dgamma and dbeta [d] float32 (None without ``weights``).  x - mean is as
    good as mean's fp32 rounding.  ``out`` (for dx) may be dy or x."""
    if _away(x, stream):
        return _there(layer_norm_grad, x, stream, dy, x, mean, rstd, gamma, weights, out)
    L = _w._lib or _w.lib()
    dt, (n, d, stride), dev = _dtype("x", x), _rows("x", x), x.device
    if dy.shape != x.shape or dy.dtype != x.dtype or dy.device != dev:
        raise ValueError("dy must be of x's shape, dtype and device")
    mean_p = _plain("mean", mean, x.shape[:-1], _F32, dev)
    rstd_p = _plain("rstd", rstd, x.shape[:-1], _F32, dev)
    gamma_p = _weight("gamma", gamma, d, x)
    dx, dx_stride = _result("out", out, x.shape, x.dtype, x)
    dgamma = dbeta = ws = None
    ws_bytes = 0
    if weights:
        dgamma, dbeta = x.new_empty((2, d), dtype=torch.float32).unbind()
        ws_bytes = L.wavernn_layer_norm_grad_workspace(n, d)
        ws = _workspace(ws_bytes, x)
    _w._check(L.wavernn_layer_norm_grad(dt, dy.data_ptr(), _rows("dy", dy)[2], x.data_ptr(), stride, n, d,
                                        _w.F32 if gamma is None else _DTYPE[gamma.dtype], gamma_p, mean_p, rstd_p,
                                        dx.data_ptr(), dx_stride, _p(dgamma), _p(dbeta), _p(ws), max(ws_bytes, 0),
                                        _raw_stream(dev.index)))
    return dx, dgamma, dbeta
