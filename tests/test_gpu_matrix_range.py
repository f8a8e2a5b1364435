"""Feed-forward blocks whose values lie far apart: nodes, tokens, hidden units and features of sizes 2^30 apart in one call, in
fp32 calls large enough for pairs of fp16 values.  Every element of every output is held to the bound that its own terms give
(`block_bound` and, for the gradient, the same roundings in `gradient_bound`).

A pair holds a value v to 2^-23 |v|, or to 2^-40 of the largest value of its row (of its column where rows are summed).  The
bounds have 40 steps of 2^-23 beside 2^-21, of the sum of the terms' sizes; a row of at least 64 normal numbers has a mean size
above 1/8 of its largest value, so 2^-40 of that largest one, for every term, is below 2^-37 of the sum of sizes.
"""
import pytest
import torch

import paper_2105_09080_b200 as pkg
import test_gpu_matrix_ops as block
from test_gpu_matrix_ops import ACT, F32, TINY, U, block_bound, normal, normal_inputs, slope, sums

pytestmark = pytest.mark.gpu

# three bfloat16 values; pairs of fp16 values, forward and gradient; the same with the weights' gradients in parts
SIZES = [(2, 90, 129, 333), (3, 1501, 700, 780), (2, 9001, 250, 500)]
FAR = 2.0 ** 30


def gradient_bound(dy, x, g, u, gate, up, down, kind):
    """[(value in 64 bits, how far an element may be off)] of dx, dgate, dup, ddown, all fp32."""
    X, DY, G, V, A, B, D = (v.double() for v in (x, dy, g, u, gate, up, down))
    t, d, f = x.shape[1], x.shape[2], g.shape[2]
    a, s = ACT[kind](G), slope(G, kind)
    dh = DY @ D
    eh = DY.abs() @ D.abs() * sums(d, F32)
    fa = 2.0 ** -21
    h, du, dg = a * V, dh * a, dh * V * s
    e_h = fa * (h.abs() + (G * V).abs())
    e_du = fa * dh.abs() * (a.abs() + G.abs()) + eh * a.abs()
    e_dg = fa * (dh * V).abs() * (1.2 + G.abs()) + eh * (V * s).abs()
    found = [(dg @ A + du @ B, sum((v.abs() + e) @ w.abs() * sums(2 * f, F32) + e @ w.abs() for v, e, w in ((dg, e_dg, A), (du, e_du, B))))]
    for v, e, o in ((dg, e_dg, X), (du, e_du, X)):
        found.append((v.mT @ o, e.mT @ o.abs() + sums(t, F32) * ((v.abs() + e).mT @ o.abs())))
    found.append((DY.mT @ h, DY.abs().mT @ e_h + sums(t, F32) * (DY.abs().mT @ (h.abs() + e_h))))
    return [(v, e + U[F32] * (v.abs() + e) + TINY[F32]) for v, e in found]


def spread(args, what, far):
    """Some nodes, tokens, hidden units or features `far` times as large as the others."""
    x, gate, up, down = (a.clone() for a in args)
    if what == "nodes":
        for a in (x, gate, up, down):
            a[1] *= far
    elif what == "inputs of a node":
        x[1] *= far
    elif what == "tokens":
        x[:, ::7] *= far
    elif what == "units":
        gate[:, 1::5] *= far
        up[:, ::5] *= far
        down[:, :, ::5] *= far
    elif what == "features":
        x[..., ::9] *= far
        down[:, ::4] *= far
    return x, gate, up, down


WHAT = ["nodes", "inputs of a node", "tokens", "units", "features"]


@pytest.mark.parametrize("far", [FAR, 1 / FAR])
@pytest.mark.parametrize("what", WHAT)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_of_values_far_apart(size, what, far):
    """Nodes whose weights are larger too are taken 2^15 apart: the products of 2^30 are too much for fp32."""
    if what in ("nodes", "units"):
        far = far ** 0.5
    args = spread(normal_inputs(*size, F32, F32, seed=40), what, far)
    for name, got, (want, bound) in zip("ygu", pkg.feed_forward_forward(*args), block_bound(*args, "silu")):
        assert ((got.double() - want).abs() <= bound).all(), name


@pytest.mark.parametrize("far", [FAR, 1 / FAR])
@pytest.mark.parametrize("what", WHAT[1:] + ["gradients of a node", "gradients of tokens", "gradients of features"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient_of_values_far_apart(size, what, far):
    """Units 2^15 apart: large and small values of gate, and of dg, lie on the summed axis of dx, where a column's small ones are
    held to 2^-40 of its largest."""
    args = normal_inputs(*size, F32, F32, seed=41)
    n, t, d, f = size
    if what == "units":
        far = far ** 0.5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(42)
    dy, g, u = normal((n, t, d), gen, F32), normal((n, t, f), gen, F32, 1.5), normal((n, t, f), gen, F32)
    if what == "gradients of a node":
        dy[1] *= far
    elif what == "gradients of tokens":
        dy[:, ::6] *= far
    elif what == "gradients of features":
        dy[..., ::9] *= far
    elif what == "units":
        u[..., ::5] *= far
    if what == "features":
        args[0][..., ::9] *= far
        args[1][..., ::7] *= far
    else:
        args = spread(args, what, far)
    x, gate, up, down = args
    got = pkg.feed_forward_backward(dy, x, g, u, gate, up, down)
    for name, a, (want, bound) in zip(("dx", "dgate", "dup", "ddown"), got, gradient_bound(dy, x, g, u, gate, up, down, "silu")):
        assert ((a.double() - want).abs() <= bound).all(), name


# 5, 3, 2 and 1 chunks of eight columns to a row; many nodes; rows that are longer than what a warp holds
NARROW = [(1, 60000, 40, 900), (1, 60001, 901, 39), (1, 100000, 20, 1050), (1, 130000, 16, 1010), (2, 130000, 8, 1010), (64, 300, 130, 900), (1, 300, 3001, 2500)]


@pytest.mark.parametrize("size", NARROW, ids=str)
def test_narrow_and_long_rows_in_pairs_are_exact(size):
    """Whole numbers, whose sums are exact in fp32 whatever their order."""
    x, gate, up, down = block.whole_inputs(*size, F32, F32, seed=50)
    gen = block.generator(51)
    dy = block.whole(x.shape, gen, F32)
    want = block.whole_forward(x, gate, up, down)
    y, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    assert all(torch.equal(a, b) for a, b in zip((y, g, u), want))
    want = [v.float() for v in block.whole_backward(dy, x, g, u, gate, up, down)]
    got = pkg.feed_forward_backward(dy, x, g, u, gate, up, down, activation="relu")
    for name, a, b in zip(("dx", "dgate", "dup", "ddown"), got, want):
        assert torch.equal(a, b), name
    pkg.token_status()


@pytest.mark.parametrize("size", NARROW, ids=str)
def test_gradient_of_narrow_and_long_rows_in_pairs(size):
    """Tokens 2^30 apart, each element within its own bound."""
    args = normal_inputs(*size, F32, F32, seed=52)
    n, t, d, f = size
    gen = block.generator(53)
    dy, g, u = normal((n, t, d), gen, F32), normal((n, t, f), gen, F32, 1.5), normal((n, t, f), gen, F32)
    dy[:, ::6] *= FAR
    got = pkg.feed_forward_backward(dy, args[0], g, u, *args[1:])
    for name, a, (want, off) in zip(("dx", "dgate", "dup", "ddown"), got, gradient_bound(dy, args[0], g, u, *args[1:], "silu")):
        assert ((a.double() - want).abs() <= off).all(), name
