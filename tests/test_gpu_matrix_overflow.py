"""Values beyond the range of a 16-bit type: they become infinities there, as a rounding makes them, and nothing else.

The second of two values that stand for one (of an fp32 weight beside 16-bit activations, of h in calls of up to eight tokens) must not
turn such an infinity into NaN.  Inputs are small whole numbers and powers of two, so that what is finite is exact."""
import pytest
import torch

import paper_2105_09080_b200 as pkg

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROWS = [1, 8, 9, 32, 33, 200]      # rows on 16 bytes and off them: every path of few tokens and the products of pieces
INF = float("inf")


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("d,f", [(16, 24), (13, 21)], ids=str)
@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
def test_gate_unit_beyond_the_range(dtype, d, f, rows):
    """h of one token and one unit is too large: infinite, and y of that token with it; the other tokens are as they were."""
    x = torch.full((1, rows, d), 0.5, dtype=dtype, device="cuda")
    x[0, 0] = 1.0
    gate, up = (torch.zeros((1, f, d), dtype=dtype, device="cuda") for _ in range(2))
    root = 2.0 ** 8 if dtype is F16 else 2.0 ** 64
    gate[0, 3, 2] = up[0, 3, 5] = root          # h = root^2 = 2^16, 2^128 of the first token, a quarter of it of the others
    down = torch.ones((1, d, f), dtype=dtype, device="cuda")
    y, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    assert (g[0, 0, 3], u[0, 0, 3]) == (root, root)
    assert (y[0, 0] == INF).all()
    assert torch.equal(y[0, 1:], torch.full_like(y[0, 1:], root * root / 4))


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("d,f", [(16, 24), (13, 21)], ids=str)
@pytest.mark.parametrize("dtype,weight", [(F16, 2.0 ** 17), (BF16, torch.finfo(F32).max)], ids=["f16", "bf16"])
def test_fp32_weight_beyond_the_range(dtype, weight, d, f, rows):
    """A finite fp32 weight that the activations' type rounds to an infinity is one; no NaN beside positive activations."""
    x = torch.ones((1, rows, d), dtype=dtype, device="cuda")
    gate, up = (torch.ones((1, f, d), device="cuda") for _ in range(2))
    down = torch.ones((1, d, f), device="cuda")
    gate[0, 3, 2], up[0, 5, 1] = weight, -weight
    _, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    want_g, want_u = (torch.full_like(g, d) for _ in range(2))
    want_g[..., 3], want_u[..., 5] = INF, -INF
    assert torch.equal(g, want_g) and torch.equal(u, want_u)
    down[0, 7, 4] = weight
    y, *_ = pkg.feed_forward_forward(x, torch.ones_like(gate), torch.ones_like(up), down, activation="relu")
    want = torch.full_like(y, f * d * d)
    want[..., 7] = INF
    assert torch.equal(y, want)
    dy = torch.ones_like(x)
    gv = torch.ones((1, rows, f), dtype=dtype, device="cuda")
    dx, *_ = pkg.feed_forward_backward(dy, x, gv, gv, gate, torch.ones_like(up), torch.ones_like(down), activation="relu")
    want = torch.full_like(dx, 2 * f * d)       # dh = d, dg = du = d, all weights one but for gate's
    want[..., 2] = INF
    assert torch.equal(dx, want)
