"""Token-block operators on small whole numbers, where every sum is exact in float32 in any grouping, so that a lost, doubled or
misplaced term of a long sum shows as a difference; and the branches that only large calls take."""
import pytest
import torch

import paper_2105_09080_b200 as pkg
from paper_2105_09080_b200.token_ops import _embedding_scratch
from test_gpu_token_ops import TYPES, U, check_forward, depth, dropped, gen, kept, near, norm_inputs, normal

pytestmark = pytest.mark.gpu


def whole(g, *shape, top=3, dtype=torch.float32):
    """Whole numbers from -top to top, no two neighbouring rows alike."""
    return torch.randint(-top, top + 1, shape, generator=g, device="cuda").to(dtype)


# ---- embedding gradient ----------------------------------------------------------------------------
def words(g, kind, nodes, rows, vocab):
    t = torch.randint(-1, vocab + 1, (nodes, rows), generator=g, device="cuda")
    if kind == "one":          # one run over all tiles
        t.fill_(vocab - 1)
    elif kind == "two":        # two runs that meet in the middle of a tile
        t[:, :rows // 2 + 3], t[:, rows // 2 + 3:] = 0, vocab - 1
    elif kind == "half":       # a run of half the tokens beside words of a few places each
        t[:, ::2] = vocab // 2
    elif kind == "steps":      # runs of 1, 2, 3, ... tokens: every way of meeting a tile's ends
        lengths = torch.arange(1, vocab, device="cuda")
        run = torch.repeat_interleave(torch.arange(vocab - 1, device="cuda"), lengths)[:rows]
        t = torch.nn.functional.pad(run, (0, rows - run.numel()), value=vocab - 1).expand(nodes, rows).contiguous()
        t = t[:, torch.randperm(rows, generator=g, device="cuda")].contiguous()
    elif kind == "none":
        t.fill_(vocab)
    return t


def grad_exact(dout, tokens, vocab):
    n, d = tokens.shape[0], dout.shape[-1]
    grad = torch.zeros((n, vocab + 1, d), dtype=torch.float64, device="cuda")
    for i in range(n):
        t = torch.where((tokens[i] < 0) | (tokens[i] >= vocab), vocab, tokens[i]).long()
        grad[i].index_add_(0, t, dout[i].double())
    return grad[:, :vocab]


def check_gradient(g, nodes, rows, d, vocab, kind, dtype):
    tokens = words(g, kind, nodes, rows, vocab)
    dout = whole(g, nodes, rows, d, dtype=dtype)
    want = grad_exact(dout, tokens, vocab)
    assert want.abs().max() < 2 ** 22
    got = pkg.embedding_backward(dout, tokens, torch.full((nodes, vocab, d), float("nan"), device="cuda"))
    assert torch.equal(got.double(), want)
    start = whole(g, nodes, vocab, d)
    got = pkg.embedding_backward(dout, tokens, start.clone(), scale=2.0, accumulate=True)
    assert torch.equal(got.double(), start.double() + 2 * want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["one", "two", "half", "steps", "spread", "none"])
@pytest.mark.parametrize("nodes,rows,d", [(1, 512, 40), (1, 513, 40), (2, 700, 9), (1, 5000, 65), (3, 4097, 24), (1, 65536, 96), (1, 65537, 33),
                                          (1, 150001, 96), (2, 66000, 1032), (1, 20011, 264)])
def test_sums_of_long_runs(dtype, kind, nodes, rows, d):
    """Up to 150001 places of one word, in one part of the token list and across parts, tiles of eight to 32 places."""
    check_gradient(gen(31), nodes, rows, d, 700 if rows > 10000 else 60, kind, dtype)


def up(v):
    return (v + 255) // 256 * 256


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["one", "two", "half", "steps", "spread"])
@pytest.mark.parametrize("nodes,rows,d,vocab", [(1, 65536, 304, 2000), (6, 65536, 56, 300), (13, 65001, 24, 300), (4, 40001, 201, 1000)])
def test_tiles_of_32_places(dtype, kind, nodes, rows, d, vocab):
    """Enough tokens and columns for the longest tiles, among them narrow rows (four places of a tile to a lane); that they
    are taken shows in the scratch's size."""
    dpad, tiles = (d + 7) // 8 * 8, (rows + 31) // 32
    want = up(nodes * rows * 8) + up(nodes * ((vocab + 31) // 32) * 4) + up(nodes * tiles * 2 * dpad * 4)
    assert _embedding_scratch(nodes, rows, d, vocab) == want
    check_gradient(gen(32), nodes, rows, d, vocab, kind, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d,vocab", [(1, 700, 8, 1500007), (2, 9000, 5, 2000003), (1, 70000, 16, 1000003)])
def test_maps_of_named_rows_in_memory(dtype, nodes, rows, d, vocab):
    """Vocabularies whose map does not fit beside the sorted entries: with 4 (14112 + 4 entries of a block) bytes taken of 227 KB,
    1.32 million rows at 700 tokens and less at more."""
    blocks = next(b for b in (1, 2, 4, 8, 16) if b == 16 or b * 1024 >= min(rows, 65536))
    of_block = -(-min(rows, 65536) // blocks)
    assert 4 * (14112 + 4 * of_block + (vocab + 31) // 32) > 227 * 1024
    for kind in ("half", "spread"):
        check_gradient(gen(33), nodes, rows, d, vocab, kind, dtype)


# ---- dropout ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d", [(3, 1001, 3304), (1, 10007, 1024), (2, 1333, 4096), (5, 20011, 104)])
def test_dropout_of_many_dense_rows(dtype, nodes, rows, d):
    """More than 148 * 8 * 1024 chunks of eight columns: four to a thread; a node's chunks are no multiple of a block's 1024."""
    chunks = rows * d // 8
    assert nodes * chunks >= 148 * 8 * 1024 and chunks % 1024
    x = normal(gen(34), nodes, rows, d, dtype=dtype)
    mask = {"k": 6, "site": 2, "node0": 3, "nodes": nodes}
    y = pkg.dropout(x, 0.3, 2 ** 40 + 9, **mask)
    keep, factor = kept(nodes, rows, d, 0.3, 2 ** 40 + 9, 6, 2, 3)
    want = dropped(x, keep, factor)
    near(y, want, 2 * U * want.abs(), dtype)
    assert (y[~keep] == 0).all()
    over = x.clone()
    assert torch.equal(pkg.dropout(over, 0.3, 2 ** 40 + 9, out=over, **mask), y)


# ---- layer norm ------------------------------------------------------------------------------------
def check_column_sums(g, nodes, rows, d, dtype, offset=0):
    """dw and db of whole numbers: z - mean and 1 / rstd are whole, so xh and every product are."""
    def activation(top):
        t = whole(g, nodes, rows, d, top=top, dtype=dtype)
        if not offset:
            return t
        wide = torch.zeros((nodes, rows, d + 11), dtype=dtype, device="cuda")
        wide[..., offset:offset + d] = t
        return wide[..., offset:offset + d]

    z, dy = activation(3), activation(2)
    mean = whole(g, nodes, rows, top=2)
    rstd = torch.randint(0, 2, (nodes, rows), generator=g, device="cuda").float() + 1
    xh = (z.double() - mean.double()[..., None]) * rstd.double()[..., None]
    want_w, want_b = (dy.double() * xh).sum(1), dy.double().sum(1)
    assert (dy.double() * xh).abs().sum(1).max() < 2 ** 24
    w = normal(g, nodes, d)
    _, _, dw, db = pkg.layer_norm_backward(dy, z, mean, rstd, w, nodes=nodes)
    assert torch.equal(dw.double(), want_w) and torch.equal(db.double(), want_b)
    acc_w, acc_b = whole(g, nodes, d), whole(g, nodes, d)
    start_w, start_b = acc_w.double(), acc_b.double()
    pkg.layer_norm_backward(dy, z, mean, rstd, w, nodes=nodes, dz=dy, p=0.5, seed=3, dweight=acc_w, dbias=acc_b, accumulate=True)
    assert torch.equal(acc_w.double(), start_w + want_w) and torch.equal(acc_b.double(), start_b + want_b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d", [(1, 100000, 64), (1, 100000, 51), (3, 30001, 128), (1, 60001, 77), (2, 20000, 256), (1, 30000, 203),
                                          (1, 20000, 512), (1, 20001, 333), (1, 12000, 768), (1, 9001, 701), (2, 9000, 1024), (1, 20000, 1003),
                                          (1, 6001, 1280), (1, 7000, 1536), (1, 5000, 1501), (1, 9000, 2048), (1, 4000, 1999), (1, 5000, 2560),
                                          (1, 3003, 2501), (1, 4001, 4096), (1, 4000, 3999), (1, 2000, 8192), (1, 2001, 7001), (1, 1501, 9001),
                                          (2, 700, 12288), (1, 33, 20000), (1, 9, 1024), (1, 8, 1024), (1, 5, 77)])
def test_column_sums_of_many_rows(dtype, nodes, rows, d):
    check_column_sums(gen(35), nodes, rows, d, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [24, 60, 200, 500, 1000, 2000, 4000, 8000, 9000])
def test_column_sums_of_many_rows_in_wider_buffers(dtype, d):
    """Inputs that are off the alignment in another way than the outputs; few rows (one block to a node) and many."""
    for rows in (5, 41, 4001):
        check_column_sums(gen(36), 1, rows, d, dtype, offset=3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d", [(12, 700, 64), (12, 131, 3000), (33, 40, 1536), (40, 20, 1501), (149, 9, 1024), (200, 33, 40), (200, 17, 77),
                                          (700, 3, 203), (300, 7, 1001), (160, 5, 2560), (1000, 2, 512), (150, 6, 8192), (151, 3, 9001)])
def test_norms_of_many_nodes(dtype, nodes, rows, d):
    """More nodes than an even share of the SMs, more nodes than SMs: blocks, masks, parameters and column sums stay a node's."""
    g = gen(37)
    x, r, w, b = norm_inputs(g, nodes, rows, d, dtype)
    mask = {"seed": 12, "k": 5, "site": 1, "node0": 7}
    check_forward(x, r, w, b, 1e-5, 0.25, mask, nodes, pkg.layer_norm_forward(x, w, b, residual=r, p=0.25, **mask), dtype)
    check_forward(x, None, w, None, 1e-5, 0.0, None, nodes, pkg.layer_norm_forward(x, w, None), dtype)
    check_column_sums(g, nodes, rows, d, dtype)
    keep, factor = kept(nodes, rows, d, 0.25, 12, 5, 1, 7)
    z, mean, rstd = x, x.double().mean(-1).float(), torch.ones((nodes, rows), device="cuda")
    dres, dx, _, _ = pkg.layer_norm_backward(r, z, mean, rstd, w, p=0.25, **mask)
    xh, h = z.double() - mean.double()[..., None], r.double() * w.double()[:, None]
    a, c = h.mean(-1, keepdim=True), (h * xh).mean(-1, keepdim=True)
    want = h - a - xh * c
    da, dc = (depth(d) + 2) * U * h.abs().mean(-1, keepdim=True), (depth(d) + 5) * U * (h * xh).abs().mean(-1, keepdim=True)
    tol = da + xh.abs() * dc + 8 * U * (h.abs() + a.abs() + (xh * c).abs()) + 2 * U * want.abs()
    near(dres, want, tol, dtype)
    near(dx, dropped(want, keep, factor), factor * tol + 2 * U * factor * want.abs(), dtype)
