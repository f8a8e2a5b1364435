"""Products whose tiles leave few over after whole waves, or are few themselves: cut between large tiles and small ones, and sums
left in parts.  Sizes are for a device of 148 multiprocessors (74 pairs); on others they run all the same."""
import pytest
import torch

import paper_2105_09080_b200 as pkg
import test_gpu_matrix_ops as block
import test_gpu_orthogonalize as orth

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32)]
# 76 tiles of 256 x 256 in the second product, four of them left over; and one node with groups of eight rows of tiles
CUT = [(19, 500, 500, 2000), (1, 18700, 200, 1500)]
# fp32 as pairs: products of 15, 24 and 30 tiles, and of 1 and 2 with long sums
PARTS = [(1, 2000, 517, 1100), (1, 9001, 250, 500), (3, 1100, 300, 1111)]


@pytest.mark.parametrize("size", CUT, ids=str)
@pytest.mark.parametrize("dtype,wtype", TYPES, ids=str)
def test_cut_between_large_and_small_tiles_is_exact(size, dtype, wtype):
    block.test_forward_of_whole_numbers_is_exact(size, dtype, wtype)
    block.test_backward_of_whole_numbers_is_exact(size, dtype, wtype)


@pytest.mark.parametrize("size", PARTS, ids=str)
def test_sums_in_parts_are_exact(size):
    """Rows on 16 bytes and off them, added to and not."""
    block.test_large_fp32_products_of_whole_numbers(size)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("size", PARTS, ids=str)
def test_gradient_of_large_fp32_blocks_against_64_bits(kind, size):
    """The bound of the smaller calls.  Two fp16 values of an array keep 2^-40 of its largest value besides 2^-24 of each: terms
    of normal numbers are on average above 2^-10 of the largest, so that is below 2^-30 of the sum of their sizes."""
    block.test_backward_against_64_bits(kind, size, F32, F32)


def test_large_fp32_blocks_in_graphs():
    """Replayed with inputs of other sizes: the powers of two belong to the replay, not to the capture."""
    size = PARTS[0]
    args, other = (block.normal_inputs(*size, F32, F32, seed=s) for s in (30, 31))
    other = [a * s for a, s in zip(other, (2.0 ** 9, 2.0 ** -5, 2.0 ** 3, 2.0 ** -12))]

    def run(a):
        y, g, u = pkg.feed_forward_forward(*a)
        return (y, g, u, *pkg.feed_forward_backward(y, a[0], g, u, *a[1:]))

    want, want_other = run(args), run(other)
    held = [a.clone() for a in args]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(held)
    for values, results in ((other, want_other), (args, want)):
        for h, v in zip(held, values):
            h.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, results))
    pkg.token_status()


# X X^T of 25 matrices of 3 tiles on and above the diagonal: cut in the last but one; of 15 of 6 and of 8 of 10: after a column
@pytest.mark.parametrize("n,r,c", [(25, 500, 1030), (15, 1030, 700), (8, 900, 1700)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_orthogonalisation_with_cut_products(n, r, c, dtype):
    """Two matrices in turn: the ones at the cut as near to the polynomial as the first."""
    pair = orth.updates(2, r, c, dtype, seed=5)
    got = pkg.orthogonalize(pair.repeat(n // 2 + 1, 1, 1)[:n].contiguous())
    delta = 2.0 ** -10 if dtype is BF16 else 2.0 ** -21
    for k in range(2):
        want, moved = orth.reference(pair[k], 5, orth.ABC, 1.0, 1e-7)
        bound = delta * moved + orth.U[dtype] * want.norm() + 2.0 ** -25 * want.numel() ** 0.5 * (dtype is F16)
        for i in range(k, n, 2):
            assert (got[i].double() - want).norm() <= bound, i
    assert torch.equal(got, pkg.orthogonalize(pair.repeat(n // 2 + 1, 1, 1)[:n].contiguous()))
    pkg.token_status()
