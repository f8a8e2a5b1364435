"""Orthogonalisation at the ends of the documented range: singular values up to 8 on the way, whose squares are 64, and a factor
c1 + c3 s^2 + c5 s^4 up to 8.

The sums of these matrices have terms of one sign, of which each matrix instruction cuts up to a step (2^-23) off.  A chunk takes 24
instructions for two values each; the first eight add rests, 2^-11 of the others, so 16 cut off its sum: 2^-19 of it beside the
2^-21 of the other tests (one value: 2^-10 as there)."""
import pytest
import torch

import paper_2105_09080_b200 as pkg
import test_gpu_orthogonalize as orth

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def leading(n, r, c, dtype, seed):
    """Matrices with one singular value that is nearly all of the norm."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    a, b = (torch.randn((n, k), generator=g, device="cuda") for k in (r, c))
    return (a[:, :, None] * b[:, None] + 2.0 ** -6 * torch.randn((n, r, c), generator=g, device="cuda")).to(dtype)


@pytest.mark.parametrize("size", [(1, 1), (60, 90), (90, 60), (200, 333), (333, 200), (520, 700)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
# 1 -> 7.38 -> 7.10; 1 -> 6 -> -6; 1 -> 2 -> 8 (all factors at most 7.5)
@pytest.mark.parametrize("steps,abc", [(2, (7.5, -0.12, 0.0)), (3, (6.2, -0.2, 0.0)), (2, (1.5, 0.45, 0.05))], ids=str)
def test_large_singular_values_on_the_way(size, dtype, steps, abc):
    m = leading(2, *size, dtype, seed=1)
    got = pkg.orthogonalize(m, steps=steps, coefficients=abc)
    assert got.isfinite().all()
    delta = 2.0 ** -10 if dtype is BF16 and min(size) > 128 else 2.0 ** -21 + 2.0 ** -19
    for i in range(2):
        want, moved = orth.reference(m[i], steps, abc, 1.0, 1e-7)
        bound = delta * moved + orth.U[dtype] * want.norm() + 2.0 ** -25 * want.numel() ** 0.5 * (dtype is F16)
        assert (got[i].double() - want).norm() <= bound


@pytest.mark.parametrize("size", [(60, 90), (200, 333)], ids=str)
@pytest.mark.parametrize("dtype", [F32, F16])
def test_a_single_large_entry(size, dtype):
    """One entry is the whole norm, so X X^T has one entry of s^2."""
    m = torch.zeros(size, dtype=dtype, device="cuda")
    m[7, 11] = -3.0
    got = pkg.orthogonalize(m, steps=2, coefficients=(7.5, -0.125, 0.0), eps=0.0)      # 1 -> 7.375 -> 5.1712
    want = torch.zeros(size, dtype=torch.float64, device="cuda")
    want[7, 11] = -(7.5 * 7.375 - 0.125 * 7.375 ** 3)
    assert ((got.double() - want).abs() <= (2.0 ** -18 + orth.U[dtype]) * want.abs()).all()
    pkg.token_status()
