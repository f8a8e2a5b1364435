"""Orthogonalisation by Newton-Schulz products on the GPU, against the polynomial of the singular values in 64 bits.

The bound: a step's rounding moves X by at most `delta` of its Frobenius norm (two fp16 values: 2^-21 for the three matrices
of a step and their sums; one: 2^-10), and an odd polynomial of a matrix's singular values moves no more than its largest
slope between the singular values' bounds times what the matrix moved.  So the error is at most the sum over the steps of
delta |X_k| times the slopes of the steps that follow, and the rounding of the result.
"""
import math

import pytest
import torch

import paper_2105_09080_b200 as pkg

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
ABC = (3.4445, -4.7750, 2.0315)
CUBIC = (1.5, -0.5, 0.0)


def updates(n, r, c, dtype, seed, scale=1e-3):
    """A few strong directions, weaker ones, and noise."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k = max(1, min(r, c) // 4)
    a = torch.randn((n, r, k), generator=g, device="cuda") * torch.arange(1, k + 1, device="cuda").float().rsqrt()
    m = a @ torch.randn((n, k, c), generator=g, device="cuda") + 0.5 * torch.randn((n, r, c), generator=g, device="cuda")
    return (m * scale).to(dtype)


def reference(m, steps, abc, scale, eps):
    """(result, bound of the error's Frobenius norm before the rounding of the result) of one matrix."""
    m = m.double()
    u, s, v = torch.linalg.svd(m, full_matrices=False)
    s = s / (s.norm() + eps)
    a, b, c = abc
    norms, slopes = [], []
    for _ in range(steps):
        norms.append(float(s.norm()))
        grid = torch.linspace(0, float(s.max()) * 1.01, 2000, dtype=torch.float64)
        slopes.append(float((a + 3 * b * grid ** 2 + 5 * c * grid ** 4).abs().max()))
        s = a * s + b * s ** 3 + c * s ** 5
    norms.append(float(s.norm()))
    moved = sum(norms[k] * math.prod(slopes[k:]) for k in range(steps)) + norms[steps]
    return scale * (u * s) @ v, abs(scale) * moved


def check(got, m, steps=5, abc=ABC, scale=1.0, eps=1e-7, base=None):
    one = m.dtype is BF16 and min(m.shape[1:]) > 128
    delta = 2.0 ** -10 if one else 2.0 ** -21
    for i in range(m.shape[0]):
        want, moved = reference(m[i], steps, abc, scale, eps)
        if base is not None:
            want = want + base[i].double()
        error = (got[i].double() - want).norm()
        assert error <= delta * moved + U[m.dtype] * want.norm() + 2.0 ** -25 * math.sqrt(want.numel()) * (m.dtype is F16), (float(error), moved)


SIZES = [(1, 1), (1, 9), (7, 1), (16, 16), (5, 300), (64, 128), (128, 64), (100, 100), (127, 129), (128, 320), (320, 128), (128, 321), (321, 100), (129, 129),
         (130, 70), (200, 333), (333, 200), (256, 256), (257, 511), (700, 1100), (1100, 700), (40, 2500), (2500, 40), (1024, 1024)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_against_64_bits(size, dtype):
    m = updates(2, *size, dtype, seed=1)
    kept = m.clone()
    got = pkg.orthogonalize(m)
    assert got.dtype is dtype and got.shape == m.shape and torch.equal(m, kept)
    check(got, m)
    assert torch.equal(pkg.orthogonalize(m), got)
    pkg.token_status()


@pytest.mark.parametrize("size", [(60, 90), (300, 180), (180, 300)], ids=str)
@pytest.mark.parametrize("steps,abc,scale", [(1, ABC, 1.0), (2, ABC, -0.3), (8, ABC, 2.0), (12, CUBIC, 1.0), (3, (1.0, 0.0, 0.0), 0.5)], ids=str)
def test_steps_coefficients_and_scale(size, steps, abc, scale):
    m = updates(3, *size, F32, seed=2)
    got = pkg.orthogonalize(m, steps=steps, coefficients=abc, scale=scale)
    check(got / scale, m, steps, abc)


def test_converges_to_an_orthogonal_matrix():
    """Enough steps of the cubic on a matrix whose singular values are alike: X X^T = 1 to a few thousand roundings."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    for r, c in ((50, 400), (400, 150)):
        x = pkg.orthogonalize(torch.randn((r, c), generator=g, device="cuda"), steps=25, coefficients=CUBIC).double()
        p = x @ x.T if r < c else x.T @ x
        assert (p - torch.eye(min(r, c), device="cuda")).abs().max() <= 2.0 ** -12


@pytest.mark.parametrize("size", [(60, 90), (200, 333)], ids=str)
def test_zero_infinite_and_extreme_matrices(size):
    m = updates(5, *size, F32, seed=4)
    clean = pkg.orthogonalize(m)
    bad = m.clone()
    bad[0] = 0
    bad[1, 3, 4] = float("inf")
    bad[2, 5, 6] = float("nan")
    got = pkg.orthogonalize(bad)
    assert (got[0] == 0).all() and got[1].isnan().all() and got[2].isnan().all()
    assert torch.equal(got[3:], clean[3:])
    assert (pkg.orthogonalize(bad, eps=0.0)[0] == 0).all()
    for factor in (1e30, 1e-30, 2.0 ** 60):     # squares past fp32's range; a power of two changes no bit
        far = pkg.orthogonalize(m * factor, eps=0.0)
        check(far, m * factor, eps=0.0)
    assert torch.equal(pkg.orthogonalize(m * 2.0 ** 60, eps=0.0), pkg.orthogonalize(m, eps=0.0))
    tiny = pkg.orthogonalize(m * 1e-9)          # eps is not small beside this norm
    check(tiny, m * 1e-9)


@pytest.mark.parametrize("size", [(24, 40), (40, 24), (130, 264), (264, 130)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("lead", [0, 3])
def test_slices_added_to(size, dtype, lead):
    """Momenta and parameters in rows of wider matrices: out = x + scale X, nothing else written; the update in its own place."""
    r, c = size
    n = 3
    m = updates(n, r, c, dtype, seed=5)
    M, X = (torch.full((n, r * c + lead + 5), float("nan"), device="cuda", dtype=dtype) for _ in range(2))
    mine, out = (t[:, lead:lead + r * c].unflatten(1, (r, c)) for t in (M, X))
    mine.copy_(m)
    base = torch.ones_like(m)
    out.copy_(base)
    assert pkg.orthogonalize(mine, scale=-0.5, out=out, accumulate=True) is out
    check(out, m, scale=-0.5, base=base)
    assert (~X.isnan()).sum() == n * r * c
    want = pkg.orthogonalize(m)
    assert torch.equal(pkg.orthogonalize(mine, out=mine), want)


def test_rows_apart():
    m = updates(2, 150, 200, F32, seed=6)
    want = pkg.orthogonalize(m)
    for pad in (1, 8):
        wide = torch.full((2, 150, 200 + pad), float("nan"), device="cuda")
        wide[..., :200] = m
        out = torch.full_like(wide, float("nan"))
        pkg.orthogonalize(wide[..., :200], out=out[..., :200])
        assert torch.equal(out[..., :200], want) and out[..., 200:].isnan().all()
    one = pkg.orthogonalize(m[0])
    assert one.shape == (150, 200) and torch.equal(one, want[0])
    shared = pkg.orthogonalize(m[:1].expand(2, 150, 200))
    assert torch.equal(shared[0], want[0]) and torch.equal(shared[1], want[0])


@pytest.mark.parametrize("size", [(64, 96), (300, 400)], ids=str)
def test_streams_and_graphs(size):
    m, o = updates(2, *size, F32, seed=7), updates(2, *size, F32, seed=8)
    want, want_o = pkg.orthogonalize(m), pkg.orthogonalize(o)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [pkg.orthogonalize(x, stream=s) for x, s in zip((m, o), streams)]
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want_o)
    held = m.clone()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(pkg.orthogonalize(held))
    held.copy_(o)
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, want_o) for x in outs)


def test_many_small_matrices():
    m = updates(1000, 12, 20, F32, seed=9)
    got = pkg.orthogonalize(m)
    check(got[::100], m[::100])
    m = updates(40, 130, 140, BF16, seed=10)
    check(pkg.orthogonalize(m)[::13], m[::13])


def test_refusals_of_the_binding():
    m = updates(2, 20, 30, F32, seed=11)
    wrong = [
        lambda: pkg.orthogonalize(m.double()), lambda: pkg.orthogonalize(m[0, 0]), lambda: pkg.orthogonalize(m[None]), lambda: pkg.orthogonalize(m.mT),
        lambda: pkg.orthogonalize(m, out=torch.empty_like(m, dtype=BF16)), lambda: pkg.orthogonalize(m, out=torch.empty_like(m[:1])),
        lambda: pkg.orthogonalize(m, out=torch.empty_like(m[0])), lambda: pkg.orthogonalize(m, out=m[:1].expand(2, 20, 30)),
        lambda: pkg.orthogonalize(m, accumulate=True), lambda: pkg.orthogonalize(m, steps=0), lambda: pkg.orthogonalize(m, coefficients=(1.0, 2.0)),
        lambda: pkg.orthogonalize(m, scale=float("nan")), lambda: pkg.orthogonalize(m, eps=-1.0), lambda: pkg.orthogonalize(m[:, :0]),
    ]
    for call in wrong:
        with pytest.raises(pkg.GpgaError):
            call()
    torch.cuda.synchronize()
