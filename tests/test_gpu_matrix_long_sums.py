"""Sums over many tokens (and over many columns) of 16-bit operands, all terms of one sign: what the matrix unit cuts off when it adds
always has the same sign too, so it must not grow with the sum's length.

What a sum may be off by, relative to it: a step (2^-23) for every matrix instruction (16 terms) that adds to one accumulator.  Those
are 32 (512 terms) where the result is fp32; the parts' sums are added in fp32, 2^-24 each.  16-bit results allow a sixteenth of
their half step: 1024 instructions for bfloat16, 256 for fp16.  In one go, 2^18 terms would be 16384 instructions."""
import pytest
import torch

import paper_2105_09080_b200 as pkg
from test_gpu_matrix_ops import U

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


INSTRUCTIONS = {F32: 32, BF16: 1024, F16: 256}


def bound(k, dtype):
    return INSTRUCTIONS[dtype] * 2.0 ** -23 + (k / 512 + 10) * 2.0 ** -24


def positive(shape, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (0.5 + torch.rand(shape, generator=g, device="cuda")).to(dtype)


def held(got, want, off, dtype):
    """A result that is `off` of itself off before its rounding lies between the roundings of what is that much smaller and larger (2^-24:
    of 64 bits to 16 over 32)."""
    off = off + 2.0 ** -24
    assert ((got >= (want * (1 - off)).to(dtype)) & (got <= (want * (1 + off)).to(dtype))).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("kind", [F32, None], ids=["fp32 gradients", "16-bit gradients"])
@pytest.mark.parametrize("rows,d,f", [(1 << 18, 64, 72), (100001, 200, 136), (60000, 520, 640)], ids=str)
def test_weights_gradients_of_many_tokens(rows, d, f, kind, dtype):
    """dh = 2^-6 times dy's first column for the first f, so that h, dg and du are exact: x is summed beside them as it is.  16-bit
    sums are below fp16's range."""
    kind = kind or dtype
    x, dy = positive((1, rows, d), dtype, 1) * 2.0 ** -6, positive((1, rows, d), dtype, 2) * 2.0 ** -6
    g = torch.ones((1, rows, f), dtype=dtype, device="cuda")
    u = positive((1, rows, f), dtype, 3) * 2.0 ** -2
    down = torch.zeros((1, d, f), dtype=dtype, device="cuda")
    down[0, 0, :] = 1.0
    gate, up = (torch.zeros((1, f, d), dtype=dtype, device="cuda") for _ in range(2))
    outs = {k: torch.empty_like(w, dtype=kind) for k, w in (("dgate", gate), ("dup", up), ("ddown", down))}
    pkg.feed_forward_backward(dy, x, g, u, gate, up, down, activation="relu", **outs)
    off = bound(rows, kind)
    du = dy[0, :, :1].double().expand(rows, f)                      # dh times g = 1
    dg = (dy[0, :, :1].double() * u[0].double()).to(dtype).double()    # fp32 holds the product of two 16-bit values
    held(outs["ddown"][0], dy[0].double().T @ u[0].double(), off, kind)
    held(outs["dup"][0], du.T @ x[0].double(), off, kind)
    held(outs["dgate"][0], dg.T @ x[0].double(), off, kind)
    pkg.token_status()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,d,f", [(40, 65536, 24), (300, 40000, 24), (40, 24, 65536), (300, 24, 40000)], ids=str)
def test_long_rows(rows, d, f, dtype):
    """Forward and dx: sums over many columns of x, of h, and of dg and du."""
    x, dy = positive((1, rows, d), dtype, 4), positive((1, rows, d), dtype, 5)
    gate, up = (positive((1, f, d), dtype, s) / d for s in (6, 7))
    down = positive((1, d, f), dtype, 8) / f
    y, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    off = bound(2 * max(d, f), dtype)
    held(g, x.double() @ gate.double().mT, off, dtype)
    held(u, x.double() @ up.double().mT, off, dtype)
    h = (g.double() * u.double())
    one = off + 2 * U[dtype] + U[dtype]      # g, u and h are rounded
    assert ((y.double() - h @ down.double().mT).abs() <= (one + U[dtype]) * (h @ down.double().mT)).all()
    dx, *_ = pkg.feed_forward_backward(dy, x, g, u, gate, up, down, activation="relu")
    dh = dy.double() @ down.double()
    want = (dh * u.double()) @ gate.double() + (dh * g.double()) @ up.double()
    assert ((dx.double() - want).abs() <= (2 * off + 2 * U[dtype]) * want).all()
    pkg.token_status()


def test_gram_matrix_of_long_rows():
    """Orthogonalisation of a wide bfloat16 matrix with one step of c1 = 0, c3 = 1: (X X^T) X, whose sums over columns are squares.
    X keeps 11 bits (2^-11 each), its mean error is far below that; A's diagonal is a sum of one sign."""
    r, c = 136, 200000
    m = positive((1, r, c), BF16, 9)
    got = pkg.orthogonalize(m, steps=1, coefficients=(0.0, 1.0, 0.0))[0].double()
    z = m[0].double() / m[0].double().norm()
    want = (z @ z.T) @ z
    e = (got - want) / want
    assert e.mean().abs() <= bound(c, F16) + 2.0 ** -12


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("wtype", [None, F32], ids=["16-bit weights", "fp32 weights"])
@pytest.mark.parametrize("rows", [4, 12, 24])
@pytest.mark.parametrize("long", [1 << 20, (1 << 20) - 3], ids=["rows on 16 bytes", "off them"])
def test_few_tokens_of_long_rows(long, rows, wtype, dtype):
    """Eight warps of a block take a part of the row each, 2^17 terms; a sum takes 4096 terms, 256 instructions, before it is added to
    the warp's.  g over a long x; y over a long h, whose values are exact."""
    wtype = wtype or dtype
    x, gate = positive((1, rows, long), dtype, 1) * 2.0 ** -5, (positive((1, 40, long), dtype, 2) * 2.0 ** -12).to(wtype)
    down = torch.zeros((1, long, 40), dtype=wtype, device="cuda")
    _, g, _ = pkg.feed_forward_forward(x, gate, gate, down, activation="relu")
    off = 256 * 2.0 ** -23 + (2 ** 17 / 4096 + 18) * 2.0 ** -24
    held(g, x.double() @ gate.double().mT, off, dtype)
    del x, gate, down
    x = torch.zeros((1, rows, 16), dtype=dtype, device="cuda")
    x[..., 0], x[..., 1] = 1.0, 2.0 ** -8
    gate, up = (torch.zeros((1, long, 16), dtype=wtype, device="cuda") for _ in range(2))
    gate[..., 0], up[..., 1] = 1.0, positive((1, long), dtype, 3).to(wtype)
    down = (positive((1, 16, long), dtype, 4) * 2.0 ** -10).to(wtype)
    y, *_ = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    h = up[..., 1].double() * 2.0 ** -8
    held(y, (h @ down[0].double().T)[:, None].expand(1, rows, 16), off, dtype)
