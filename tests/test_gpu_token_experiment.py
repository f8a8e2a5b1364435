"""The token model on the GPU: every node's gradient row against automatic differentiation in 64 bits, and a short
training run by Algorithm 1."""
import pytest
import torch

import paper_2105_09080_b200 as pkg
from paper_2105_09080_b200 import token_experiment as te
from test_gpu_token_ops import U, kept

pytestmark = pytest.mark.gpu


def test_gradient_rows_against_automatic_differentiation():
    """float32 activations: relative error of each gradient row's parts a few hundred roundings (sums of up to 96 terms,
    three products deep) of the part's norm."""
    n, T, V, D, p, k = 4, 96, 40, 24, 0.2, 7
    m = te.TokenModel(n, V, D, pkg.GPGA_TOPO_RING, 4, 5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    m.X[:, :m.d] += 0.1 * torch.randn((n, m.d), generator=gen, device="cuda")
    before, cur, target = te.batch(n, T, V, k, 1)
    m.G.fill_(float("nan"))
    loss = m.gradient(k, before, cur, target, p)
    X = m.X.double().requires_grad_()
    A, Bt, Ct, w, b = m.slices(X)
    keep, factor = kept(n, T, D, p, m.seed, k, 0)
    node = torch.arange(n, device="cuda")[:, None]
    z = Bt[node, before] + A[node, cur] * keep * factor
    y = torch.nn.functional.layer_norm(z, (D,), eps=1e-5) * w[:, None] + b[:, None]
    logits = y @ Ct.transpose(1, 2)
    want = torch.stack([torch.nn.functional.cross_entropy(logits[i], target[i]) for i in range(n)])
    assert ((loss.double() - want).abs() <= 1000 * U * want).all()
    want.sum().backward()
    for got, ref in zip(m.slices(m.G), m.slices(X.grad)):
        for i in range(n):
            assert (got[i].double() - ref[i]).norm() <= 1000 * U * ref[i].norm()
    m.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_run(dtype):
    """All methods learn the common rule (the loss of a uniform guess is ln 64 = 4.16); parallel SGD's rows stay equal, the
    others' differ between averages."""
    runs = {}
    for name, topology, H in te.METHODS:
        out = te.train(name, topology, H, n=8, T=256, vocab=64, dim=64, iters=150, every=50, gamma=1.0, dtype=dtype)
        runs[name] = out["trajectory"]
        assert out["trajectory"][-1]["average_loss"] < 2.5
    assert runs["parallel SGD"][-1]["consensus"] == 0.0
    assert runs["Gossip SGD, ring"][-1]["consensus"] > 0.0
