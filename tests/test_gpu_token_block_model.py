"""The token model with a gated feed-forward block: every node's gradient row against automatic differentiation in 64 bits, the
local update with orthogonalised momenta, and that a run of both works with the mixing."""
import math

import pytest
import torch

import paper_2105_09080_b200 as pkg
from paper_2105_09080_b200 import token_experiment as te
from test_gpu_token_ops import U, kept

pytestmark = pytest.mark.gpu


def model(dtype=torch.float32, update="plain", n=4, V=40, D=24, hidden=56, seed=5):
    m = te.TokenModel(n, V, D, pkg.GPGA_TOPO_RING, 4, seed, dtype=dtype, hidden=hidden, update=update)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    m.X[:, :m.d] += 0.1 * torch.randn((n, m.d), generator=gen, device="cuda")
    return m


def reference(m, before, cur, target, p, k):
    """(losses, gradient of their sum) in 64 bits."""
    n, T = cur.shape
    X = m.X.double().requires_grad_()
    A, Bt, Ct, w, b = m.slices(X)
    gate, up, down = m.matrices(X)
    keep, factor = kept(n, T, m.dim, p, m.seed, k, 0)
    node = torch.arange(n, device="cuda")[:, None]
    z = Bt[node, before] + A[node, cur] * keep * factor
    y = torch.nn.functional.layer_norm(z, (m.dim,), eps=1e-5) * w[:, None] + b[:, None]
    y = y + (torch.nn.functional.silu(y @ gate.mT) * (y @ up.mT)) @ down.mT
    logits = y @ Ct.mT
    losses = torch.stack([torch.nn.functional.cross_entropy(logits[i], target[i]) for i in range(n)])
    losses.sum().backward()
    return losses.detach(), X.grad


def test_gradient_rows_against_automatic_differentiation():
    """float32: relative error of each part of a gradient row a few hundred roundings (sums of up to 96 terms, seven products
    deep) of the part's norm."""
    m = model()
    p, k = 0.2, 7
    batch = te.batch(m.n, 96, m.vocab, k, 1)
    m.G.fill_(float("nan"))
    loss = m.gradient(k, *batch, p)
    want, grad = reference(m, *batch, p, k)
    assert ((loss.double() - want).abs() <= 1000 * U * want).all()
    for got, ref in zip((*m.slices(m.G), *m.matrices(m.G)), (*m.slices(grad), *m.matrices(grad))):
        for i in range(m.n):
            assert (got[i].double() - ref[i]).norm() <= 2000 * U * ref[i].norm()
    m.close()


@pytest.mark.parametrize("dtype,u", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
def test_gradient_of_16_bit_activations(dtype, u):
    """The parts of a row are off by some roundings of the activations (a dozen values are rounded on the way to each, and
    their errors meet in sums); the reference sees none of them."""
    m = model(dtype)
    batch = te.batch(m.n, 96, m.vocab, 0, 1)
    m.gradient(0, *batch, 0.0)
    _, grad = reference(m, *batch, 0.0, 0)
    for got, ref in zip((*m.slices(m.G), *m.matrices(m.G)), (*m.slices(grad), *m.matrices(grad))):
        for i in range(m.n):
            assert (got[i].double() - ref[i]).norm() <= 16 * u * ref[i].norm()
    m.close()


def test_orthogonal_update():
    """One local update without mixing: m = mu m + g, x - gamma_m sqrt(max(1, r / c)) times the orthogonalised m."""
    m = te.TokenModel(3, 24, 16, pkg.GPGA_TOPO_NONE, 0, 5, hidden=40, update="orthogonal")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    m.G.copy_(torch.randn(m.G.shape, generator=gen, device="cuda"))
    m.M.copy_(torch.randn(m.M.shape, generator=gen, device="cuda"))
    X, M = m.X.double().clone(), m.M.double().clone()
    m.step(0, 0.1)
    M = m.momentum * M + m.G[:, m.first_matrix:m.d].double()
    assert ((m.M.double() - M).abs() <= 4 * U * (M.abs() + m.G.abs().max())).all()
    assert ((m.X[:, :m.first_matrix].double() - (X - 0.1 * m.G)[:, :m.first_matrix]).abs() <= 4 * U * (1 + X.abs() + m.G.abs())[:, :m.first_matrix]).all()
    for before, mom, after in zip(m.matrices(X), m.matrices(m.M, 0), m.matrices(m.X)):
        for i in range(m.n):
            u, s, v = torch.linalg.svd(mom[i].double(), full_matrices=False)
            s = s / (s.norm() + 1e-7)
            for _ in range(5):
                s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
            want = before[i] - m.matrix_gamma * math.sqrt(max(1.0, mom.shape[1] / mom.shape[2])) * (u * s) @ v
            # 485 = the polynomial's slope at zero to the fifth power: the most that a rounding of the start can grow
            assert (after[i].double() - want).norm() <= m.matrix_gamma * 485 * 2.0 ** -20 + 2 * U * want.norm()
    m.close()


@pytest.mark.parametrize("update", ["plain", "orthogonal"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_a_run_works(update, dtype):
    """Gradient, update and mixing for some iterations: everything stays finite, the rows meet at the global average."""
    out = te.train("Gossip-PGA, ring", pkg.GPGA_TOPO_RING, 4, n=4, T=64, vocab=32, dim=32, iters=12, every=4, gamma=0.5, dtype=dtype, hidden=72, update=update)
    assert out["hidden"] == 72 and out["update"] == update
    for point in out["trajectory"]:
        assert all(math.isfinite(point[key]) for key in ("loss", "average_loss", "consensus"))
    assert out["trajectory"][0]["consensus"] == 0.0
    pkg.token_status()


def test_refusals():
    with pytest.raises(ValueError):
        te.TokenModel(2, 8, 8, pkg.GPGA_TOPO_RING, 0, 1, update="orthogonal")
    with pytest.raises(ValueError):
        te.TokenModel(2, 8, 8, pkg.GPGA_TOPO_RING, 0, 1, hidden=8, update="other")


def test_the_model_without_a_block_is_as_it_was():
    """Same row length, same first rows, same gradient with and without the new arguments."""
    a, b = te.TokenModel(2, 24, 16, pkg.GPGA_TOPO_RING, 0, 5), te.TokenModel(2, 24, 16, pkg.GPGA_TOPO_RING, 0, 5, hidden=0, update="plain")
    assert a.d == b.d == 3 * 24 * 16 + 2 * 16 and torch.equal(a.X, b.X) and a.M is None
    batch = te.batch(2, 32, 24, 0, 1)
    a.gradient(0, *batch, 0.1)
    b.gradient(0, *batch, 0.1)
    assert torch.equal(a.G, b.G)
    a.close()
    b.close()
