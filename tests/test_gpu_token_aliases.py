"""Layer norm whose output replaces its input: what is returned for the backward call is z, whatever the output overwrites."""
import pytest
import torch

import paper_2105_09080_b200 as pkg
from test_gpu_token_ops import EPS, SHAPES, TYPES, U, check_forward, depth, gen, near, norm_inputs, normal

pytestmark = pytest.mark.gpu


def check_returned(x, w, b, dy, over, got, dtype):
    """y, z and the statistics against the definition on x; the gradient that they lead to against its definition in 64
    bits, with the roundings of xh (2), h (1), the row sums and the four operations of g."""
    nodes, rows, d = x.shape
    y, z, mean, rstd = got
    assert y is over
    assert torch.equal(z.view_as(x), x)
    check_forward(x, None, w, b, 1e-5, 0.0, None, nodes, got, dtype)
    g, dx, dw, db = pkg.layer_norm_backward(dy, z, mean, rstd, w)
    assert dx is g
    W, s = w.double()[:, None], rstd.double()[..., None]
    xh = (x.double() - mean.double()[..., None]) * s
    h = dy.double() * W
    mh, mhx = h.mean(-1, keepdim=True), (h * xh).mean(-1, keepdim=True)
    want = s * (h - mh - xh * mhx)
    dmh, dmhx = (depth(d) + 2) * U * h.abs().mean(-1, keepdim=True), (depth(d) + 5) * U * (h * xh).abs().mean(-1, keepdim=True)
    near(g, want, s * (dmh + xh.abs() * dmhx + 8 * U * (h.abs() + mh.abs() + (xh * mhx).abs())) + 2 * U * want.abs(), dtype)
    near(dw, (dy.double() * xh).sum(1), (rows + 3) * U * (dy.double() * xh).abs().sum(1), torch.float32)
    near(db, dy.double().sum(1), rows * U * dy.double().abs().sum(1), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d", SHAPES)
def test_backward_after_a_norm_over_its_input(dtype, nodes, rows, d):
    g = gen(21)
    x, _, w, b = norm_inputs(g, nodes, rows, d, dtype)
    dy = normal(g, nodes, rows, d, dtype=dtype)
    over = x.clone()
    check_returned(x, w, b, dy, over, pkg.layer_norm_forward(over, w, b, out=over), dtype)
    # z wanted in the input's own place, beside an output of its own: nothing to copy, nothing lost
    y, z, _, _ = pkg.layer_norm_forward(over.copy_(x), w, b, z=over)
    assert z is over and torch.equal(z, x) and y is not over


def test_backward_after_a_norm_over_a_view_of_its_input():
    """The output as another tensor on the same memory, dense and inside a wider buffer."""
    g = gen(22)
    for d in (24, 77, 512, 1001):
        x, _, w, b = norm_inputs(g, 2, 9, d, torch.float32)
        dy = normal(g, 2, 9, d)
        wide = normal(g, 2, 9, d + 5)
        wide[..., 2:2 + d] = x
        over = wide[..., 2:2 + d]
        check_returned(x, w, b, dy, over, pkg.layer_norm_forward(wide[..., 2:2 + d], w, b, out=over), torch.float32)
        dense = x.clone()
        over = dense.view(2, 9, d)
        check_returned(x, w, b, dy, over, pkg.layer_norm_forward(dense, w, b, out=over), torch.float32)
