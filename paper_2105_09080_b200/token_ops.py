"""Token-block operators on torch CUDA tensors: embedding lookup and its gradient, dropout from the library's
counter-based generator, layer norm (with the residual sum and the dropout in front of it) and its gradient.

Argument marshalling only, as in ``binding``: every operator is one C entry of include/gpga.h, which has the formulas.
They work node by node.  Parameters and their gradients are float32 and may be slices of the state matrix X (n, ld) and
of a gradient matrix of the same shape: ``X[:, a:a + V * d].unflatten(1, (V, d))`` is a table argument.  Activations are
float32, bfloat16 or float16; all of one call have one type.  An activation (..., d) is taken as vectors of d values;
with ``nodes`` nodes the first nodes-th part of the vectors belongs to node 0 and so on.  Vectors may lie apart (a slice
of a wider buffer), evenly spaced.

Outputs, statistics and scratch are allocated unless they are given.  Calls are asynchronous on ``stream`` (default: the
current one), allocate through torch's allocator only and can be captured in a CUDA graph.  With a ``stream`` other than
the current one the new tensors belong to that stream and the given ones are marked as used there; ordering the two
streams is the caller's part.
"""
from __future__ import annotations

import contextlib

import torch

from .binding import GPGA_ERR_INVALID_ARG, GPGA_OK, GpgaError, lib

GPGA_DTYPE_F32, GPGA_DTYPE_BF16, GPGA_DTYPE_F16 = 0, 1, 2
_DTYPE = {torch.float32: GPGA_DTYPE_F32, torch.bfloat16: GPGA_DTYPE_BF16, torch.float16: GPGA_DTYPE_F16}
_TOKEN_BYTES = {torch.int32: 4, torch.int64: 8}
_nothing = contextlib.nullcontext()


def _bad(text):
    raise GpgaError(GPGA_ERR_INVALID_ARG, text)


def _check(st):
    if st != GPGA_OK:
        raise GpgaError(st, lib().gpga_last_error(None).decode())


def _spacing(t):
    """Distance in elements between neighbouring vectors of ``t`` (..., d)."""
    if t.is_contiguous():
        return t.shape[-1]
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        _bad(f"the last dimension must be dense, got strides {t.stride()}")
    ld = None
    step = 0
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = step = stride
        elif stride != step:
            _bad(f"vectors must be evenly spaced, got shape {tuple(t.shape)} with strides {t.stride()}")
        step *= size
    return t.shape[-1] if ld is None else ld


def _act(t, what, like, dtype=None):
    """Pointer and spacing of an activation that must have the shape (and type) of ``like``; None gives NULL."""
    if t is None:
        return None, 0
    if t.dtype != (dtype or like.dtype) or t.shape != like.shape or t.device != like.device:
        _bad(f"{what}: got {tuple(t.shape)} {t.dtype} on {t.device}, want {tuple(like.shape)} {dtype or like.dtype} on {like.device}")
    return t.data_ptr(), _spacing(t)


def _stats(t, what, like):
    """Pointer of a dense float32 vector of one value per row of ``like``."""
    if t.dtype != torch.float32 or t.numel() * like.shape[-1] != like.numel() or not t.is_contiguous() or t.device != like.device:
        _bad(f"{what} must be contiguous float32, one value per row, on {like.device}")
    return t.data_ptr()


def _params(t, what, nodes, d, device):
    """Pointer and node stride of a float32 parameter (d,) or (nodes, d); None gives NULL."""
    if t is None:
        return None, 0
    if t.dtype != torch.float32 or t.device != device or t.shape[-1] != d or t.numel() != nodes * d or t.dim() > 2 \
            or (t.stride(-1) != 1 and d > 1):
        _bad(f"{what}: got {tuple(t.shape)} {t.dtype} on {t.device}, want dense float32 rows of ({nodes}, {d}) on {device}")
    return t.data_ptr(), (t.stride(0) if t.dim() == 2 and nodes > 1 else d)


def _table(t, what, tokens):
    """(nodes, vocab, d, row stride, node stride) of a table (vocab, d) or (nodes, vocab, d)."""
    if t.dtype != torch.float32 or t.dim() not in (2, 3) or not t.is_cuda or (t.stride(-1) != 1 and t.shape[-1] > 1):
        _bad(f"{what} must be a float32 CUDA tensor (vocab, d) or (nodes, vocab, d) with dense rows, got {tuple(t.shape)} {t.dtype}")
    if tokens.dtype not in _TOKEN_BYTES or not tokens.is_contiguous() or tokens.device != t.device:
        _bad(f"tokens must be contiguous int32 or int64 on {t.device}, got {tokens.dtype} on {tokens.device}")
    if t.dim() == 2:
        return 1, t.shape[0], t.shape[1], max(t.stride(0), t.shape[1]) if t.shape[0] == 1 else t.stride(0), 0
    if tokens.dim() < 1 or tokens.shape[0] != t.shape[0]:
        _bad(f"tokens must be (nodes, ...) with nodes = {t.shape[0]}, got {tuple(tokens.shape)}")
    n, vocab, d = t.shape
    ld = max(t.stride(1), d) if vocab == 1 else t.stride(1)
    return n, vocab, d, ld, (max(t.stride(0), (vocab - 1) * ld + d) if n == 1 else t.stride(0))


def _on(stream, *tensors):
    """Stream pointer of a launch; the tensors' device must be current.  Tensors used on a stream that is not the
    current one are marked for the allocator."""
    index = tensors[0].device.index
    if torch.cuda.current_device() != index:
        _bad(f"tensors live on {tensors[0].device} but cuda:{torch.cuda.current_device()} is current")
    if stream is None:
        return torch.cuda.current_stream(index).cuda_stream
    s = torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream
    if s.cuda_stream != torch.cuda.current_stream(index).cuda_stream:
        for t in tensors:
            if t is not None:
                t.record_stream(s)
    return s.cuda_stream


def _owner(stream):
    """Where new tensors of a call are allocated: the launch's stream."""
    if stream is None:
        return _nothing
    return torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)


def _scratch(need, scratch, device):
    if scratch is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if scratch.device != device or not scratch.is_contiguous():
        _bad(f"scratch must be contiguous on {device}")
    return scratch


def _rows(x, nodes):
    """Activation checks: (rows per node, d, dtype code)."""
    dtype = _DTYPE.get(x.dtype)
    if dtype is None or not x.is_cuda or x.dim() < 1 or x.shape[-1] < 1:
        _bad(f"activations must be float32, bfloat16 or float16 CUDA tensors (..., d), got {tuple(x.shape)} {x.dtype} on {x.device}")
    d = x.shape[-1]
    vectors = x.numel() // d
    if nodes < 1 or vectors % nodes:
        _bad(f"{vectors} vectors do not split over {nodes} nodes")
    return vectors // nodes, d, dtype


def embedding_forward(table, tokens, scale=1.0, dtype=None, out=None, stream=None):
    """out[..., :] = scale * table[tokens[...], :] (gpga_embedding_forward).

    ``table`` (V, d) with ``tokens`` of any shape, or (n, V, d) with tokens (n, ...): node i looks up in table[i].
    Tokens outside [0, V) give zero rows.  ``dtype``: of the new output (default float32); ``out``: write here.
    """
    nodes, vocab, d, ldt, node_ldt = _table(table, "table", tokens)
    if out is None:
        with _owner(stream):
            out = torch.empty(tokens.shape + (d,), dtype=dtype or torch.float32, device=table.device)
    elif out.shape != tokens.shape + (d,) or out.device != table.device or (dtype is not None and out.dtype != dtype):
        _bad(f"out: got {tuple(out.shape)} {out.dtype}, want {tuple(tokens.shape) + (d,)} on {table.device}")
    code = _DTYPE.get(out.dtype)
    if code is None:
        _bad(f"out must be float32, bfloat16 or float16, got {out.dtype}")
    _check(lib().gpga_embedding_forward(table.data_ptr(), ldt, node_ldt, tokens.data_ptr(), _TOKEN_BYTES[tokens.dtype],
                                        out.data_ptr(), _spacing(out), code, nodes, tokens.numel() // nodes, d, vocab,
                                        scale, _on(stream, table, tokens, out)))
    return out


def embedding_backward(dout, tokens, grad_table, scale=1.0, accumulate=False, scratch=None, stream=None):
    """grad_table[v, :] = scale * (sum of dout[t, :] over the t with tokens[t] = v), or added to it (gpga_embedding_backward).

    ``grad_table`` has the table's shape, float32, and is returned; without ``accumulate`` all of its rows are written.
    """
    nodes, vocab, d, ldg, node_ldg = _table(grad_table, "grad_table", tokens)
    code = _DTYPE.get(dout.dtype)
    if code is None or dout.shape != tokens.shape + (d,) or dout.device != grad_table.device:
        _bad(f"dout: got {tuple(dout.shape)} {dout.dtype} on {dout.device}, want {tuple(tokens.shape) + (d,)} on {grad_table.device}")
    rows = tokens.numel() // nodes
    with _owner(stream):
        scratch = _scratch(lib().gpga_embedding_scratch_bytes(nodes, rows, d, vocab), scratch, dout.device)
    _check(lib().gpga_embedding_backward(dout.data_ptr(), _spacing(dout), code, tokens.data_ptr(), _TOKEN_BYTES[tokens.dtype],
                                         grad_table.data_ptr(), ldg, node_ldg, nodes, rows, d, vocab, scale, accumulate,
                                         scratch.data_ptr(), scratch.numel() * scratch.element_size(),
                                         _on(stream, dout, tokens, grad_table, scratch)))
    return grad_table


def dropout(x, p, seed, k=0, site=0, node0=0, nodes=1, out=None, stream=None):
    """x with each element dropped with probability p, the others divided by the probability of staying (gpga_dropout).

    The mask is a function of (seed, k, site, node, row of the node, column); the gradient is the same call on the
    output's gradient.  ``out`` may be ``x``.
    """
    rows, d, dtype = _rows(x, nodes)
    if out is None:
        with _owner(stream):
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    yp, ldy = _act(out, "out", x)
    _check(lib().gpga_dropout(x.data_ptr(), _spacing(x), yp, ldy, dtype, nodes, rows, d, p, seed, k, site, node0,
                              _on(stream, x, out)))
    return out


def _nodes_of(weight, nodes):
    if nodes is not None:
        return nodes
    return weight.shape[0] if weight is not None and weight.dim() == 2 else 1


def layer_norm_forward(x, weight, bias, eps=1e-5, residual=None, p=0.0, seed=0, k=0, site=0, node0=0, nodes=None,
                       out=None, z=None, mean=None, rstd=None, stream=None):
    """Layer norm of z = residual + dropout(x) (gpga_layer_norm_forward): returns (y, z, mean, rstd).

    ``weight`` and ``bias``: (d,), (nodes, d) or None.  z is ``x`` itself where there is neither a residual nor
    dropout.  mean and rstd: one float32 per row.  What the backward call wants is z, mean and rstd.
    """
    nodes = _nodes_of(weight, nodes)
    rows, d, dtype = _rows(x, nodes)
    mixed = residual is not None or p > 0
    with _owner(stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if z is None and mixed:
            z = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if mean is None:
            mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        if rstd is None:
            rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    wp, ldw = _params(weight, "weight", nodes, d, x.device)
    bp, ldb = _params(bias, "bias", nodes, d, x.device)
    if bp is not None and wp is not None and ldb != ldw:
        _bad("weight and bias must have one node stride")
    rp, ldr = _act(residual, "residual", x)
    yp, ldy = _act(out, "out", x)
    zp, ldz = _act(z, "z", x)
    _check(lib().gpga_layer_norm_forward(x.data_ptr(), _spacing(x), rp, ldr, wp, bp, ldw if wp is not None else ldb, yp, ldy,
                                         zp, ldz, _stats(mean, "mean", x), _stats(rstd, "rstd", x), dtype, nodes, rows, d, eps,
                                         p, seed, k, site, node0,
                                         _on(stream, x, residual, weight, bias, out, z, mean, rstd)))
    return out, (z if z is not None else x), mean, rstd


def layer_norm_backward(dy, z, mean, rstd, weight, dz=None, p=0.0, seed=0, k=0, site=0, node0=0, nodes=None,
                        dresidual=None, dx=None, dweight=None, dbias=None, accumulate=False, scratch=None, stream=None):
    """Gradient of ``layer_norm_forward`` (gpga_layer_norm_backward): returns (dresidual, dx, dweight, dbias).

    ``dz``: gradient that reaches z past the norm.  dx is dresidual itself where p = 0.  dweight and dbias are sums over
    each node's rows, added to what the given tensors hold with ``accumulate``; without a weight they are None unless
    given.
    """
    nodes = _nodes_of(weight, nodes)
    rows, d, dtype = _rows(z, nodes)
    if accumulate and (dweight is None or dbias is None):
        _bad("accumulate wants dweight and dbias")
    with _owner(stream):
        if dresidual is None:
            dresidual = torch.empty(z.shape, dtype=z.dtype, device=z.device)
        if dx is None and p > 0:
            dx = torch.empty(z.shape, dtype=z.dtype, device=z.device)
        if weight is not None:
            if dweight is None:
                dweight = torch.empty(weight.shape, dtype=torch.float32, device=z.device)
            if dbias is None:
                dbias = torch.empty(weight.shape, dtype=torch.float32, device=z.device)
        scratch = _scratch(lib().gpga_layer_norm_scratch_bytes(nodes, rows, d), scratch, z.device)
    wp, ldw = _params(weight, "weight", nodes, d, z.device)
    dwp, lddw = _params(dweight, "dweight", nodes, d, z.device)
    dbp, lddb = _params(dbias, "dbias", nodes, d, z.device)
    if dwp is not None and dbp is not None and lddw != lddb:
        _bad("dweight and dbias must have one node stride")
    dyp, lddy = _act(dy, "dy", z)
    ep, lde = _act(dz, "dz", z)
    gp, ldg = _act(dresidual, "dresidual", z)
    xp, ldx = _act(dx, "dx", z)
    _check(lib().gpga_layer_norm_backward(dyp, lddy, z.data_ptr(), _spacing(z), ep, lde, _stats(mean, "mean", z),
                                          _stats(rstd, "rstd", z), wp, ldw, gp, ldg, xp, ldx, dwp, dbp,
                                          lddw if dwp is not None else lddb, accumulate, dtype, nodes, rows, d, p, seed, k,
                                          site, node0, scratch.data_ptr(), scratch.numel() * scratch.element_size(),
                                          _on(stream, z, dy, dz, mean, rstd, weight, dresidual, dx, dweight, dbias, scratch)))
    return dresidual, (dx if dx is not None else dresidual), dweight, dbias
