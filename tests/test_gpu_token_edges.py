"""Token-block operators at the edges of what their definitions say."""
import numpy as np
import pytest
import torch

import paper_2105_09080_b200 as pkg
from test_gpu_token_ops import U, check_forward, depth, gen, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [7, 77, 640, 1000, 1001, 1024, 5000, 9001, 20000])
def test_layer_norm_of_constant_rows(d):
    """A constant row's mean is as good as its sum: off by at most the additions' rounding, and by one product's and its
    correction's.  What remains of the row is that error times 1 / sqrt(eps), the variance at most its square."""
    g = gen(41)
    values = torch.tensor([0.36159506, 3.0, -0.1, 1e-3, 1234.567, -7e4, 0.0], device="cuda")
    x = values[:, None].expand(-1, d).contiguous()
    w, b = 1 + 0.2 * normal(g, d), 0.3 * normal(g, d)
    eps = float(np.float32(1e-5))
    c = values.double()[:, None]
    off = (depth(d) + 2) * U * c.abs()
    for weight, bias in ((w, b), (w, None), (None, None)):
        y, z, mean, rstd = pkg.layer_norm_forward(x, weight, bias, eps=1e-5)
        W = weight.double().abs() if weight is not None else 1.0
        B = bias.double() if bias is not None else torch.zeros(d, dtype=torch.float64, device="cuda")
        assert z is x and ((mean.double()[:, None] - c).abs() <= off).all()
        assert (rstd.double()[:, None] <= eps ** -0.5 * (1 + 4 * U)).all()
        assert (rstd.double()[:, None] >= (eps + off * off) ** -0.5 * (1 - 8 * U)).all()
        assert ((y.double() - B).abs() <= W * off * eps ** -0.5 * (1 + 8 * U) + 2 * U * B.abs()).all()
        assert torch.equal(y[-1].double(), B.expand(d))


@pytest.mark.parametrize("d", [24, 77, 1024])
def test_norms_without_a_weight(d):
    """A bias of every node alone, gradients of parameters that the norm does not multiply by, nothing to add up: the
    gradients are those of a weight of ones."""
    g = gen(42)
    n, T = 3, 9
    x, b, dy = normal(g, n, T, d), normal(g, n, d), normal(g, n, T, d)
    ones = torch.ones((n, d), device="cuda")
    y, z, mean, rstd = pkg.layer_norm_forward(x, None, b)
    check_forward(x, None, None, b, 1e-5, 0.0, None, n, (y, z, mean, rstd), torch.float32)
    assert torch.equal(y, pkg.layer_norm_forward(x, None, b, nodes=n)[0])
    want = pkg.layer_norm_backward(dy, x, mean, rstd, ones)
    start = normal(g, n, d)
    for names in (("dweight",), ("dbias",), ("dweight", "dbias")):
        given = {k: torch.full((n, d), float("nan"), device="cuda") for k in names}
        got = pkg.layer_norm_backward(dy, x, mean, rstd, None, **given)
        assert torch.equal(got[0], want[0])
        for at, name in ((2, "dweight"), (3, "dbias")):
            assert got[at] is given.get(name) and (got[at] is None or torch.equal(got[at], want[at]))
        more = {k: start.clone() for k in names}
        got = pkg.layer_norm_backward(dy, x, mean, rstd, None, accumulate=True, **more)
        for at, name in ((2, "dweight"), (3, "dbias")):
            assert got[at] is None or torch.equal(got[at], start + want[at])
    got = pkg.layer_norm_backward(dy, x, mean, rstd, None, accumulate=True)
    assert torch.equal(got[0], want[0]) and got[2] is None and got[3] is None
    for given in ({}, {"dweight": start.clone()}, {"dbias": start.clone()}):      # with a weight both are written
        with pytest.raises(pkg.GpgaError):
            pkg.layer_norm_backward(dy, x, mean, rstd, ones, accumulate=True, **given)


def test_tensors_that_require_gradients_are_taken_for_their_values():
    """No call takes part in automatic differentiation: the same values with and without, and nothing behind them."""
    g = gen(43)
    table, w, x = normal(g, 11, 40), normal(g, 40), normal(g, 6, 40)
    tokens = torch.randint(0, 11, (6,), generator=g, device="cuda")

    def calls(table, w, x):
        y, z, mean, rstd = pkg.layer_norm_forward(x, w, w, residual=x, p=0.1, seed=3)
        return [pkg.embedding_forward(table, tokens), pkg.dropout(x, 0.3, 5), y, z, mean, rstd,
                *pkg.layer_norm_backward(x, z, mean, rstd, w, p=0.1, seed=3)]

    want = calls(table, w, x)
    got = calls(*(torch.nn.Parameter(t) for t in (table, w, x)))
    assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(got, want))
