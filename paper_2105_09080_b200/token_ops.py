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

These are plain functions, outside automatic differentiation: tensors that require gradients are taken for their values,
what comes back has no graph behind it, and a model calls the ``_backward`` functions itself (as ``token_experiment``
does, or inside a ``torch.autograd.Function`` of its own).
"""
from __future__ import annotations

import functools
import struct

import torch

from .binding import GPGA_ERR_INVALID_ARG, GPGA_OK, GpgaError, lib

GPGA_DTYPE_F32, GPGA_DTYPE_BF16, GPGA_DTYPE_F16 = 0, 1, 2
_DTYPE = {torch.float32: GPGA_DTYPE_F32, torch.bfloat16: GPGA_DTYPE_BF16, torch.float16: GPGA_DTYPE_F16}
_TOKEN_BYTES = {torch.int32: 4, torch.int64: 8}

# The argument structs of include/gpga.h, packed in one go (a small call's time is its marshalling): Q device pointer or
# seed, q size or stride, d double.
ARGS = {
    "gpga_embedding_forward": struct.Struct("=3Q9qd"),
    "gpga_embedding_backward": struct.Struct("=4Q11qd"),
    "gpga_dropout": struct.Struct("=2Q6qdQ3q"),
    "gpga_layer_norm_forward": struct.Struct("=8Q9q2dQ3q"),
    "gpga_layer_norm_backward": struct.Struct("=11Q13qdQ3q"),
}

_current_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream


def _bad(text):
    raise GpgaError(GPGA_ERR_INVALID_ARG, text)


@functools.lru_cache(maxsize=None)
def _entry(name):
    """What calls a C entry on the current stream of a device with the members of its argument struct."""
    fn, pack, L = getattr(lib(), name), ARGS[name].pack, lib()

    def call(device, *members):
        if device != _current_device():
            _bad(f"tensors live on cuda:{device} but cuda:{_current_device()} is current")
        try:
            args = pack(*members)
        except struct.error as e:
            _bad(f"argument out of range: {e}")
        st = fn(args, _raw_stream(device))
        if st != GPGA_OK:
            raise GpgaError(st, L.gpga_last_error(None).decode())
    return call


@functools.lru_cache(maxsize=4096)
def _embedding_scratch(nodes, rows, d, vocab):
    return lib().gpga_embedding_scratch_bytes(nodes, rows, d, vocab)


@functools.lru_cache(maxsize=4096)
def _norm_scratch(nodes, rows, d):
    return lib().gpga_layer_norm_scratch_bytes(nodes, rows, d)


def _on_stream(fn, args):
    """The same call with ``stream`` as the current stream; tensors of another stream are marked for the allocator."""
    stream = args.pop("stream")
    s = torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream
    if s.cuda_stream != torch.cuda.current_stream(s.device).cuda_stream:
        for t in args.values():
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(s)
    with torch.cuda.stream(s):
        return fn(**args)


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


def _same(t, what, shape, dtype, device, d):
    """Spacing of an activation that must have this shape and type."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _bad(f"{what}: got {tuple(t.shape)} {t.dtype} on {t.device}, want {tuple(shape)} {dtype} on cuda:{device}")
    return d if t.is_contiguous() else _spacing(t)


def _stats(t, what, vectors, device):
    """Pointer of a dense float32 vector of one value per row."""
    if t.dtype is not torch.float32 or t.numel() != vectors or t.get_device() != device or not t.is_contiguous():
        _bad(f"{what} must be contiguous float32 on cuda:{device}, {vectors} values (one per row)")
    return t.data_ptr()


def _params(t, what, nodes, d, device):
    """Node stride of a float32 parameter (d,) or (nodes, d)."""
    if t.dtype is not torch.float32 or t.get_device() != device or t.numel() != nodes * d or t.dim() not in (1, 2) or t.shape[-1] != d:
        _bad(f"{what}: got {tuple(t.shape)} {t.dtype} on {t.device}, want float32 ({nodes}, {d}) on cuda:{device}")
    if t.is_contiguous():
        return d
    if t.stride(-1) != 1 and d > 1:
        _bad(f"{what}: rows must be dense, got strides {t.stride()}")
    return t.stride(0) if nodes > 1 else d


def _table(t, what, tokens):
    """(device, nodes, vocab, d, row stride, node stride) of a table (vocab, d) or (nodes, vocab, d)."""
    shape, device = t.shape, t.get_device()
    if t.dtype is not torch.float32 or len(shape) not in (2, 3) or device < 0 or 0 in shape:
        _bad(f"{what} must be a float32 CUDA tensor (vocab, d) or (nodes, vocab, d), got {tuple(shape)} {t.dtype} on {t.device}")
    if tokens.dtype not in _TOKEN_BYTES or tokens.get_device() != device or not tokens.is_contiguous():
        _bad(f"tokens must be contiguous int32 or int64 on {t.device}, got {tokens.dtype} on {tokens.device}")
    vocab, d = shape[-2:]
    nodes = shape[0] if len(shape) == 3 else 1
    if len(shape) == 3 and (tokens.dim() < 1 or tokens.shape[0] != nodes):
        _bad(f"tokens must be (nodes, ...) with nodes = {nodes}, got {tuple(tokens.shape)}")
    if t.is_contiguous():
        return device, nodes, vocab, d, d, vocab * d
    stride = t.stride()
    if stride[-1] != 1 and d > 1:
        _bad(f"{what}: rows must be dense, got strides {stride}")
    ld = stride[-2] if vocab > 1 else d
    return device, nodes, vocab, d, ld, stride[0] if nodes > 1 else vocab * ld


def _vectors(x, nodes):
    """Checks of the activation that a call goes by: (shape, type, its code, device, d, rows per node)."""
    dtype, shape, device = x.dtype, x.shape, x.get_device()
    code = _DTYPE.get(dtype)
    if code is None or device < 0 or not shape or not shape[-1]:
        _bad(f"activations must be float32, bfloat16 or float16 CUDA tensors (..., d), got {tuple(shape)} {dtype} on {x.device}")
    d = shape[-1]
    vectors = x.numel() // d
    if nodes < 1 or vectors % nodes:
        _bad(f"{vectors} vectors do not split over {nodes} nodes")
    return shape, dtype, code, device, d, vectors // nodes


def _like(x):
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _scratch(scratch, need, like, device):
    """(tensor, pointer, bytes) of a call's scratch: the given tensor, or a new one where the call needs any."""
    if scratch is None:
        if not need:
            return None, 0, 0
        scratch = like.new_empty(need, dtype=torch.uint8)
    elif scratch.get_device() != device or not scratch.is_contiguous():
        _bad(f"scratch must be contiguous on cuda:{device}")
    return scratch, scratch.data_ptr(), scratch.nbytes


def embedding_forward(table, tokens, scale=1.0, dtype=None, out=None, stream=None):
    """out[..., :] = scale * table[tokens[...], :] (gpga_embedding_forward).

    ``table`` (V, d) with ``tokens`` of any shape, or (n, V, d) with tokens (n, ...): node i looks up in table[i].
    Tokens outside [0, V) give zero rows.  ``dtype``: of the new output (default float32); ``out``: write here.
    """
    if stream is not None:
        return _on_stream(embedding_forward, locals())
    device, nodes, vocab, d, ldt, node_ldt = _table(table, "table", tokens)
    shape = tokens.shape + (d,)
    if out is None:
        out = table.new_empty(shape, dtype=dtype or torch.float32)
    code = _DTYPE.get(out.dtype)
    if code is None:
        _bad(f"out must be float32, bfloat16 or float16, got {out.dtype}")
    ldo = _same(out, "out", shape, dtype or out.dtype, device, d)
    _entry("gpga_embedding_forward")(device, table.data_ptr(), tokens.data_ptr(), out.data_ptr(), ldt, node_ldt, ldo,
                                     _TOKEN_BYTES[tokens.dtype], code, nodes, tokens.numel() // nodes, d, vocab, scale)
    return out


def embedding_backward(dout, tokens, grad_table, scale=1.0, accumulate=False, scratch=None, stream=None):
    """grad_table[v, :] = scale * (sum of dout[t, :] over the t with tokens[t] = v), or added to it (gpga_embedding_backward).

    ``grad_table`` has the table's shape, float32, and is returned; without ``accumulate`` all of its rows are written.
    """
    if stream is not None:
        return _on_stream(embedding_backward, locals())
    device, nodes, vocab, d, ldg, node_ldg = _table(grad_table, "grad_table", tokens)
    code = _DTYPE.get(dout.dtype)
    if code is None:
        _bad(f"dout must be float32, bfloat16 or float16, got {dout.dtype}")
    ldo = _same(dout, "dout", tokens.shape + (d,), dout.dtype, device, d)
    rows = tokens.numel() // nodes
    scratch, scratch_p, scratch_bytes = _scratch(scratch, _embedding_scratch(nodes, rows, d, vocab), dout, device)
    _entry("gpga_embedding_backward")(device, dout.data_ptr(), tokens.data_ptr(), grad_table.data_ptr(), scratch_p,
                                      scratch_bytes, ldo, ldg, node_ldg, _TOKEN_BYTES[tokens.dtype], code, nodes, rows, d,
                                      vocab, accumulate, scale)
    return grad_table


def dropout(x, p, seed, k=0, site=0, node0=0, nodes=1, out=None, stream=None):
    """x with each element dropped with probability p, the others divided by the probability of staying (gpga_dropout).

    The mask is a function of (seed, k, site, node, row of the node, column); the gradient is the same call on the
    output's gradient.  ``out`` may be ``x``.
    """
    if stream is not None:
        return _on_stream(dropout, locals())
    shape, dtype, code, device, d, rows = _vectors(x, nodes)
    if out is None:
        out = _like(x)
    ldy = _same(out, "out", shape, dtype, device, d)
    _entry("gpga_dropout")(device, x.data_ptr(), out.data_ptr(), d if x.is_contiguous() else _spacing(x), ldy, code, nodes, rows,
                           d, p, seed, k, site, node0)
    return out


def _nodes_of(nodes, *params):
    """The given number of nodes, or that of the first parameter that is there."""
    if nodes is not None:
        return nodes
    for t in params:
        if t is not None:
            return t.shape[0] if t.dim() == 2 else 1
    return 1


def layer_norm_forward(x, weight, bias, eps=1e-5, residual=None, p=0.0, seed=0, k=0, site=0, node0=0, nodes=None,
                       out=None, z=None, mean=None, rstd=None, stream=None):
    """Layer norm of z = residual + dropout(x) (gpga_layer_norm_forward): returns (y, z, mean, rstd).

    ``weight`` and ``bias``: (d,), (nodes, d) or None; without ``nodes`` they say how many there are.  z is ``x`` itself
    where there is neither a residual nor dropout, unless y replaces it (``out`` in x's place): then z is a tensor of its
    own.  mean and rstd: one float32 per row.  What the backward call wants is z, mean and rstd.
    """
    if stream is not None:
        return _on_stream(layer_norm_forward, locals())
    nodes = _nodes_of(nodes, weight, bias)
    shape, dtype, code, device, d, rows = _vectors(x, nodes)
    if out is None:
        out = _like(x)
    if z is None and (residual is not None or p > 0 or out.data_ptr() == x.data_ptr()):
        z = _like(x)
    if mean is None:
        mean = x.new_empty(shape[:-1], dtype=torch.float32)
    if rstd is None:
        rstd = x.new_empty(shape[:-1], dtype=torch.float32)
    wp = bp = rp = zp = ldw = ldr = ldz = 0
    if weight is not None:
        wp, ldw = weight.data_ptr(), _params(weight, "weight", nodes, d, device)
    if bias is not None:
        bp, ldb = bias.data_ptr(), _params(bias, "bias", nodes, d, device)
        if weight is None:
            ldw = ldb
        elif ldb != ldw:
            _bad("weight and bias must have one node stride")
    if residual is not None:
        rp, ldr = residual.data_ptr(), _same(residual, "residual", shape, dtype, device, d)
    if z is not None:
        zp, ldz = z.data_ptr(), _same(z, "z", shape, dtype, device, d)
    _entry("gpga_layer_norm_forward")(device, x.data_ptr(), rp, wp, bp, out.data_ptr(), zp,
                                      _stats(mean, "mean", nodes * rows, device), _stats(rstd, "rstd", nodes * rows, device),
                                      d if x.is_contiguous() else _spacing(x), ldr, ldw,
                                      _same(out, "out", shape, dtype, device, d), ldz, code, nodes, rows, d, eps, p, seed, k,
                                      site, node0)
    return out, (x if z is None else z), mean, rstd


def layer_norm_backward(dy, z, mean, rstd, weight, dz=None, p=0.0, seed=0, k=0, site=0, node0=0, nodes=None,
                        dresidual=None, dx=None, dweight=None, dbias=None, accumulate=False, scratch=None, stream=None):
    """Gradient of ``layer_norm_forward`` (gpga_layer_norm_backward): returns (dresidual, dx, dweight, dbias).

    ``dz``: gradient that reaches z past the norm.  dx is dresidual itself where p = 0.  dweight and dbias are sums over
    each node's rows, added to what the given tensors hold with ``accumulate`` (which wants both beside a weight);
    without a weight they are None unless given.
    """
    if stream is not None:
        return _on_stream(layer_norm_backward, locals())
    nodes = _nodes_of(nodes, weight, dweight, dbias)
    shape, dtype, code, device, d, rows = _vectors(z, nodes)
    if accumulate and weight is not None and (dweight is None or dbias is None):
        _bad("accumulate wants dweight and dbias")
    if dresidual is None:
        dresidual = _like(z)
    if dx is None and p > 0:
        dx = _like(z)
    wp = dwp = dbp = ep = xp = ldw = lddw = lde = ldx = 0
    if weight is not None:
        wp, ldw = weight.data_ptr(), _params(weight, "weight", nodes, d, device)
        if dweight is None:
            dweight = weight.new_empty(weight.shape)
        if dbias is None:
            dbias = weight.new_empty(weight.shape)
    if dweight is not None:
        dwp, lddw = dweight.data_ptr(), _params(dweight, "dweight", nodes, d, device)
    if dbias is not None:
        dbp, lddb = dbias.data_ptr(), _params(dbias, "dbias", nodes, d, device)
        if dweight is None:
            lddw = lddb
        elif lddb != lddw:
            _bad("dweight and dbias must have one node stride")
    if dz is not None:
        ep, lde = dz.data_ptr(), _same(dz, "dz", shape, dtype, device, d)
    if dx is not None:
        xp, ldx = dx.data_ptr(), _same(dx, "dx", shape, dtype, device, d)
    scratch, scratch_p, scratch_bytes = _scratch(scratch, _norm_scratch(nodes, rows, d), z, device)
    _entry("gpga_layer_norm_backward")(device, dy.data_ptr(), z.data_ptr(), ep, _stats(mean, "mean", nodes * rows, device),
                                       _stats(rstd, "rstd", nodes * rows, device), wp, dresidual.data_ptr(), xp, dwp, dbp,
                                       scratch_p, scratch_bytes, _same(dy, "dy", shape, dtype, device, d),
                                       d if z.is_contiguous() else _spacing(z), lde, ldw,
                                       _same(dresidual, "dresidual", shape, dtype, device, d), ldx, lddw, accumulate, code,
                                       nodes, rows, d, p, seed, k, site, node0)
    return dresidual, (dresidual if dx is None else dx), dweight, dbias
