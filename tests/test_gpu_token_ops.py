"""Token-block operators (embedding lookup, dropout, layer norm and their gradients) on the GPU against plain forms
in 64 bits.

Tolerances come from the operations' rounding: u = 2^-24 is the fp32 unit roundoff, EPS[t] the one rounding to the
output type; a sum of m fp32 terms in any grouping of depth s is off by at most s u sum |terms|.  DEPTH bounds the depth
of a row sum here: at most 8 * ceil(d / 8192) sequential additions per thread in the widest loops tested plus 64 for the
registers of one thread, shuffles and warps.
"""
import math

import numpy as np
import pytest
import torch

import paper_2105_09080_b200 as pkg

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}   # spacing of subnormals
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def depth(d):
    return 64 + 8 * math.ceil(d / 8192)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def near(got, want, tol, dtype):
    """|got - want| <= tol + the one rounding of want to dtype, element by element; NaN and infinities equal."""
    want = want.double()
    got = got.double()
    ok = (got - want).abs() <= tol * (1 + 2.0 ** -8) + EPS[dtype] * (1 + 2.0 ** -8) * want.abs() + TINY[dtype]
    ok |= (got == want) | (got.isnan() & want.isnan())
    assert ok.all(), f"{(~ok).sum().item()} of {ok.numel()} off, first at {(~ok).nonzero()[0].tolist()}, " \
                     f"max {(got - want).abs()[~ok].max().item()}"


# ---- references ------------------------------------------------------------------------------------
def philox(ctr, key):
    """Philox4x32-10 in numpy on four uint64 arrays that hold 32-bit words."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, dtype=np.uint64) for x in ctr]
    k0, k1 = key
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def kept(nodes, rows, d, p, seed, k, site, node0=0):
    """(nodes, rows, d) truth values and the factor, from the definition."""
    q = math.floor(65536 * p + 0.5)
    groups = -(-d // 8)
    c0 = (np.arange(rows)[:, None] * groups + np.arange(groups)).astype(np.uint64)
    out = np.empty((nodes, rows, groups, 8), dtype=np.uint32)
    for i in range(nodes):
        w = philox([c0, np.full_like(c0, node0 + i), np.full_like(c0, k), np.full_like(c0, 0x40000000 + site)],
                   (seed & 0xFFFFFFFF, seed >> 32))
        for j in range(8):
            out[i, :, :, j] = (w[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)
    keep = torch.from_numpy(out.reshape(nodes, rows, groups * 8)[..., :d].copy().astype(np.int64) >= q)
    return keep.cuda(), (65536.0 / (65536 - q) if q < 65536 else 0.0)


def dropped(x, keep, factor):
    return torch.where(keep, x.double() * factor, torch.zeros((), dtype=torch.float64, device="cuda"))


def norm_reference(z, w, b, eps):
    mean = z.mean(-1, keepdim=True)
    var = (z - mean).square().mean(-1, keepdim=True)
    rstd = (var + eps) ** -0.5
    return (z - mean) * rstd * w + b, mean, rstd, var


# ---- lookup ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d,vocab", [(1, 1, 1, 1), (1, 1, 1024, 500), (3, 17, 8, 5), (2, 33, 257, 1000), (1, 300, 72, 70000),
                                                (5, 9, 1028, 33), (2, 5, 12001, 50)])
def test_lookup(dtype, nodes, rows, d, vocab):
    g = gen(1)
    table = normal(g, nodes, vocab, d)
    tokens = torch.randint(-2, vocab + 2, (nodes, rows), generator=g, device="cuda", dtype=torch.int32 if d % 2 else torch.int64)
    out = pkg.embedding_forward(table, tokens, scale=0.7, dtype=dtype)
    valid = (tokens >= 0) & (tokens < vocab)
    rowsel = table[torch.arange(nodes, device="cuda")[:, None], tokens.long().clamp(0, vocab - 1)].double()
    want = torch.where(valid[..., None], rowsel * float(np.float32(0.7)), torch.zeros((), dtype=torch.float64, device="cuda"))
    near(out, want, U * want.abs(), dtype)


def test_lookup_in_slices_of_the_state_matrix():
    """Tables inside rows of X at an odd place, output vectors inside a wider buffer, tokens of three dimensions."""
    g = gen(2)
    n, V, d, ld = 3, 40, 24, 40 * 24 + 37
    X = normal(g, n, ld)
    table = X[:, 5:5 + V * d].unflatten(1, (V, d))
    tokens = torch.randint(0, V, (n, 4, 6), generator=g, device="cuda")
    wide = torch.full((n, 4, 6, 50), 7.0, device="cuda", dtype=torch.bfloat16)
    out = pkg.embedding_forward(table, tokens, out=wide[..., 3:3 + d])
    want = torch.stack([table[i][tokens[i]] for i in range(n)])
    assert torch.equal(out, want.bfloat16())
    assert (wide[..., :3] == 7).all() and (wide[..., 3 + d:] == 7).all()
    one = pkg.embedding_forward(table[1], tokens[1])
    assert torch.equal(one, table[1][tokens[1]])


# ---- its gradient ----------------------------------------------------------------------------------
def grad_reference(dout, tokens, vocab, scale):
    """(grad, bound): the sums in float64 and the bound of the fp32 sums' error."""
    n, d = tokens.shape[0], dout.shape[-1]
    grad = torch.zeros((n, vocab + 1, d), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(grad)
    count = torch.zeros((n, vocab + 1), dtype=torch.float64, device="cuda")
    for i in range(n):
        t = tokens[i].reshape(-1).long()
        t = torch.where((t < 0) | (t >= vocab), torch.full_like(t, vocab), t)
        e = dout[i].reshape(-1, d).double()
        grad[i].index_add_(0, t, e)
        mag[i].index_add_(0, t, e.abs())
        count[i].index_add_(0, t, torch.ones_like(t, dtype=torch.float64))
    # additions in sequence: at most the number of terms (8 per join of partial sums are among them), and the scaling
    bound = (count[..., None] + 2) * U * mag * abs(scale)
    return (grad * scale)[:, :vocab], bound[:, :vocab]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d,vocab", [(1, 1, 1, 1), (1, 1, 64, 300), (2, 16, 8, 5), (3, 17, 65, 1000), (1, 700, 257, 30),
                                                (2, 1025, 1024, 77), (1, 5000, 40, 300000), (4, 9, 1100, 65536), (1, 20011, 136, 3),
                                                (2, 512, 1030, 40), (3, 513, 20, 40), (1, 40000, 264, 5000), (2, 600, 2052, 900), (1, 9000, 8, 70000),
                                                (1, 700, 9, 1000003), (3, 17000, 40, 50)])
def test_lookup_gradient(dtype, nodes, rows, d, vocab):
    g = gen(3)
    tokens = torch.randint(-1, vocab + 1, (nodes, rows), generator=g, device="cuda", dtype=torch.int64 if d % 2 else torch.int32)
    tokens[:, : rows // 3] = vocab // 2      # a token that spans tiles
    dout = normal(g, nodes, rows, d, dtype=dtype)
    grad = torch.full((nodes, vocab, d), float("nan"), device="cuda")
    scale = float(np.float32(1.3))
    got = pkg.embedding_backward(dout, tokens, grad, scale=scale)
    assert got is grad
    want, bound = grad_reference(dout, tokens, vocab, scale)
    near(got, want, bound + U * want.abs(), torch.float32)
    named = torch.zeros((nodes, vocab), dtype=torch.bool, device="cuda")
    for i in range(nodes):
        named[i][tokens[i][(tokens[i] >= 0) & (tokens[i] < vocab)].long()] = True
    assert (got[~named] == 0).all()
    again = pkg.embedding_backward(dout, tokens, torch.empty_like(grad), scale=scale)
    assert torch.equal(again, got)           # the same bits in every run
    start = normal(g, nodes, vocab, d)
    more = pkg.embedding_backward(dout, tokens, start.clone(), scale=scale, accumulate=True)
    near(more, start.double() + want, bound + U * (want.abs() + start.abs().double()) * 2, torch.float32)
    assert torch.equal(more[~named], start[~named])


def test_lookup_gradient_of_one_word_and_of_many_tokens():
    """A run of thousands of equal tokens over many tiles; more tokens than one cluster sorts; no valid token at all."""
    g = gen(4)
    for rows, vocab in ((65536, 2000), (150001, 2000)):
        d = 96
        dout = normal(g, 1, rows, d, dtype=torch.bfloat16)
        for kind in ("one", "half", "spread", "none"):
            tokens = torch.randint(0, vocab, (1, rows), generator=g, device="cuda")
            if kind == "one":
                tokens.fill_(vocab - 1)
            if kind == "half":
                tokens[:, ::2] = 0
            if kind == "none":
                tokens.fill_(-1)
            got = pkg.embedding_backward(dout, tokens, torch.full((1, vocab, d), float("nan"), device="cuda"))
            want, bound = grad_reference(dout, tokens, vocab, 1.0)
            near(got, want, bound, torch.float32)


def test_lookup_gradient_without_tokens():
    grad = torch.full((2, 9, 20), 3.0, device="cuda")
    tokens = torch.empty((2, 0), dtype=torch.int64, device="cuda")
    dout = torch.empty((2, 0, 20), device="cuda")
    pkg.embedding_backward(dout, tokens, grad, accumulate=True)
    assert (grad == 3).all()
    pkg.embedding_backward(dout, tokens, grad)
    assert (grad == 0).all()
    assert pkg.embedding_forward(grad, tokens).shape == (2, 0, 20)


def test_lookup_gradient_into_slices_of_the_gradient_matrix():
    """Rows of G at an odd place, dout inside a wider buffer; nothing beside the slices is written.  Non-finite
    gradients reach the rows of their tokens and no others."""
    g = gen(5)
    n, V, d = 3, 50, 33
    G = torch.full((n, 11 + V * d + 6), 5.0, device="cuda")
    part = G[:, 11:11 + V * d].unflatten(1, (V, d))
    wide = normal(g, n, 70, d + 9)
    wide[0, 3, 4] = float("inf")
    wide[2, 5, 6] = float("nan")
    tokens = torch.randint(0, V, (n, 70), generator=g, device="cuda")
    dout = wide[..., 2:2 + d]
    pkg.embedding_backward(dout, tokens, part)
    want, bound = grad_reference(dout, tokens, V, 1.0)
    bound = torch.nan_to_num(bound, nan=0.0, posinf=0.0)
    near(part, want, bound, torch.float32)
    assert (G[:, :11] == 5).all() and (G[:, 11 + V * d:] == 5).all()


def test_lookup_offsets_beyond_32_bits():
    V, d = 70001, 32768                       # 2.3e9 elements
    table = torch.zeros((V, d), device="cuda")
    g = gen(6)
    tokens = torch.tensor([V - 1, 0, 65600, V - 1], device="cuda")
    table[V - 1] = normal(g, d)
    table[65600] = normal(g, d)
    out = pkg.embedding_forward(table, tokens)
    assert torch.equal(out, table[tokens])
    table.fill_(2.0)
    dout = normal(g, 4, d)
    pkg.embedding_backward(dout, tokens, table)
    assert torch.equal(table[V - 1], dout[0] + dout[3]) and torch.equal(table[65600], dout[2])
    assert (table[65601:V - 1:97] == 0).all() and torch.equal(table[0], dout[1])


# ---- dropout ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
@pytest.mark.parametrize("nodes,rows,d", [(1, 1, 1), (1, 19, 333), (3, 7, 64), (2, 5, 1000), (4, 3, 8200)])
def test_dropout(dtype, p, nodes, rows, d):
    x = normal(gen(7), nodes, rows, d, dtype=dtype)
    seed, k, site, node0 = 0x123456789ABCDEF0, 2 ** 32 - 3, 2 ** 30 - 1, 5
    y = pkg.dropout(x, p, seed, k=k, site=site, node0=node0, nodes=nodes)
    keep, factor = kept(nodes, rows, d, p, seed, k, site, node0)
    want = dropped(x, keep, factor)
    near(y, want, 2 * U * want.abs(), dtype)
    assert (y[~keep] == 0).all()
    inplace = x.clone()
    assert torch.equal(pkg.dropout(inplace, p, seed, k=k, site=site, node0=node0, nodes=nodes, out=inplace), y)


def test_dropout_of_views_and_special_values():
    """A slice of a wider buffer at an odd place gives what a dense copy gives; NaN and infinities vanish where they are
    dropped and stay where they are kept; the masks of sites, iterations, nodes and seeds differ."""
    wide = normal(gen(8), 30, 200, dtype=torch.bfloat16)
    x = wide[:, 3:131]
    y = pkg.dropout(x, 0.4, 99)
    assert torch.equal(y, pkg.dropout(x.contiguous(), 0.4, 99))
    keep, _ = kept(1, 30, 128, 0.4, 99, 0, 0)
    for value in (float("inf"), float("-inf"), float("nan"), torch.finfo(torch.float32).min):
        z = pkg.dropout(torch.full((1, 30, 128), value, device="cuda"), 0.4, 99)
        assert (z[~keep] == 0).all()
        assert z[keep].isnan().all() if math.isnan(value) else torch.isinf(z[keep]).all()
    ones = torch.ones((1, 64, 256), device="cuda")
    base = pkg.dropout(ones, 0.5, 1)
    others = [pkg.dropout(ones, 0.5, 2), pkg.dropout(ones, 0.5, 1 + 2 ** 40), pkg.dropout(ones, 0.5, 1, k=1),
              pkg.dropout(ones, 0.5, 1, site=1), pkg.dropout(ones, 0.5, 1, node0=1)]
    n = ones.numel()
    for o in others:      # independent masks agree in half the places: 6 standard deviations of a binomial
        assert abs((o == base).float().mean().item() - 0.5) < 6 * 0.5 / math.sqrt(n)
    assert abs((base != 0).float().mean().item() - 0.5) < 6 * 0.5 / math.sqrt(n)
    both = pkg.dropout(torch.ones((2, 64, 256), device="cuda"), 0.5, 1, nodes=2)
    assert torch.equal(both[0], base[0]) and torch.equal(both[1], others[4][0])


# ---- layer norm ------------------------------------------------------------------------------------
SHAPES = [(1, 1, 1), (1, 3, 7), (2, 70, 121), (1, 33, 128), (3, 9, 700), (1, 19, 1208), (2, 7, 1501), (1, 6, 2560), (2, 5, 8), (1, 40, 64), (3, 11, 65), (2, 9, 200), (1, 300, 256), (2, 13, 512), (1, 17, 1000),
          (3, 50, 1023), (2, 33, 1024), (1, 6, 2048), (2, 3, 2056), (1, 4, 4100), (1, 5, 8192), (1, 3, 9001), (2, 2, 16392)]


def norm_inputs(g, nodes, rows, d, dtype):
    x = (normal(g, nodes, rows, d) * 1.5 + normal(g, nodes, rows, 1)).to(dtype)
    r = normal(g, nodes, rows, d, dtype=dtype)
    return x, r, 1 + 0.2 * normal(g, nodes, d), 0.3 * normal(g, nodes, d)


def check_forward(x, r, w, b, eps, p, mask, nodes, got, dtype):
    y, z, mean, rstd = got
    d = x.shape[-1]
    rows = x.numel() // d // nodes
    if p > 0:
        keep, factor = kept(nodes, rows, d, p, mask["seed"], mask["k"], mask["site"], mask["node0"])
        zx = dropped(x.view(nodes, rows, d), keep, factor)
    else:
        zx = x.view(nodes, rows, d).double()
    rd = r.view(nodes, rows, d).double() if r is not None else torch.zeros_like(zx)
    zr = zx + rd
    W = w.double().view(-1, 1, d) if w is not None else torch.ones((1, 1, d), dtype=torch.float64, device="cuda")
    B = b.double().view(-1, 1, d) if b is not None else torch.zeros((1, 1, d), dtype=torch.float64, device="cuda")
    want, m, s, var = norm_reference(zr, W, B, eps)
    dz = 3 * U * (zx.abs() + rd.abs())                       # dropout's factor and product, the sum
    dm = depth(d) * U * zr.abs().mean(-1, keepdim=True) + dz.mean(-1, keepdim=True)
    # of the variance: its own sum, twice the covariance with dz, the square of the mean's error
    dv = depth(d) * U * var + 2 * (dz * (zr - m).abs()).mean(-1, keepdim=True) + dm * dm + dm * dz.mean(-1, keepdim=True) * 2
    ds = (0.5 * dv / (var + eps) + 4 * U) * s
    dy = W.abs() * (s * (dz + dm) + (zr - m).abs() * ds + 3 * U * s * (zr - m).abs()) + U * (want.abs() + B.abs())
    near(y.view(nodes, rows, d), want, 2 * dy, dtype)        # twice: products of two errors
    near(mean.view(nodes, rows, 1), m, 2 * dm, torch.float32)
    near(rstd.view(nodes, rows, 1), s, 2 * ds, torch.float32)
    near(z.view(nodes, rows, d), zr, dz, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d", SHAPES)
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (True, 0.25)])
def test_layer_norm_forward(dtype, nodes, rows, d, residual, p):
    x, r, w, b = norm_inputs(gen(9), nodes, rows, d, dtype)
    r = r if residual else None
    mask = {"seed": 77 + 2 ** 35, "k": 12, "site": 4, "node0": 1}
    got = pkg.layer_norm_forward(x, w, b, eps=1e-5, residual=r, p=p, **mask)
    assert residual or p > 0 or got[1] is x
    check_forward(x, r, w, b, 1e-5, p, mask, nodes, got, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nodes,rows,d", SHAPES + [(1, 4000, 72), (3, 1001, 264)])
@pytest.mark.parametrize("dz,p", [(False, 0.0), (True, 0.0), (True, 0.25)])
def test_layer_norm_backward(dtype, nodes, rows, d, dz, p):
    g = gen(10)
    z, e, w, _ = norm_inputs(g, nodes, rows, d, dtype)
    dy = normal(g, nodes, rows, d, dtype=dtype)
    zd = z.double()
    mean = zd.mean(-1).float()
    rstd = ((zd - zd.mean(-1, keepdim=True)).square().mean(-1) + 1e-5).rsqrt().float()
    mask = {"seed": 5, "k": 3, "site": 9, "node0": 2}
    dres, dx, dw, db = pkg.layer_norm_backward(dy, z, mean, rstd, w, dz=e if dz else None, p=p, **mask)
    assert (dx is dres) == (p == 0)
    W, s = w.double()[:, None], rstd.double()[..., None]
    xh = (zd - mean.double()[..., None]) * s
    h = dy.double() * W
    mh, mhx = h.mean(-1, keepdim=True), (h * xh).mean(-1, keepdim=True)
    E = e.double() if dz else torch.zeros_like(zd)
    want = s * (h - mh - xh * mhx) + E
    # roundings of xh (2), h (1), the row sums, and the four operations of g
    dmh, dmhx = (depth(d) + 2) * U * h.abs().mean(-1, keepdim=True), (depth(d) + 5) * U * (h * xh).abs().mean(-1, keepdim=True)
    tol = s * (dmh + xh.abs() * dmhx + 8 * U * (h.abs() + mh.abs() + (xh * mhx).abs())) + 2 * U * (want.abs() + E.abs())
    near(dres, want, tol, dtype)
    if p > 0:
        keep, factor = kept(nodes, rows, d, p, mask["seed"], mask["k"], mask["site"], mask["node0"])
        near(dx, dropped(want, keep, factor), factor * tol + 2 * U * factor * want.abs(), dtype)
    # column sums: at most all rows in sequence, three roundings per term
    near(dw, (dy.double() * xh).sum(1), (rows + 3) * U * (dy.double() * xh).abs().sum(1), torch.float32)
    near(db, dy.double().sum(1), rows * U * dy.double().abs().sum(1), torch.float32)
    again = pkg.layer_norm_backward(dy, z, mean, rstd, w, dz=e if dz else None, p=p, **mask)
    assert all(torch.equal(a, b) for a, b in zip(again, (dres, dx, dw, db)))
    start_w, start_b = normal(g, nodes, d), normal(g, nodes, d)
    acc_w, acc_b = start_w.clone(), start_b.clone()
    pkg.layer_norm_backward(dy, z, mean, rstd, w, dz=e if dz else None, p=p, dweight=acc_w, dbias=acc_b, accumulate=True, **mask)
    near(acc_w, start_w.double() + dw.double(), 2 * U * (start_w.abs() + dw.abs()).double(), torch.float32)
    near(acc_b, start_b.double() + db.double(), 2 * U * (start_b.abs() + db.abs()).double(), torch.float32)


def test_layer_norm_gradient_against_differences():
    """Central differences in 64 bits of sum(c y) + sum(e z), y and z as the forward call defines them, against the
    backward call in fp32: by x, the residual, the weight and the bias."""
    g = gen(11)
    nodes, rows, d, p, eps = 2, 3, 11, 0.3, 1e-3
    x, r, w, b = norm_inputs(g, nodes, rows, d, torch.float32)
    c, e = normal(g, nodes, rows, d), normal(g, nodes, rows, d)
    mask = {"seed": 8, "k": 1, "site": 2, "node0": 0}
    y, z, mean, rstd = pkg.layer_norm_forward(x, w, b, eps=eps, residual=r, p=p, **mask)
    dres, dx, dw, db = pkg.layer_norm_backward(c, z, mean, rstd, w, dz=e, p=p, **mask)
    keep, factor = kept(nodes, rows, d, p, 8, 1, 2)

    def f(x, r, w, b):
        z = dropped(x, keep, factor) + r
        return (c.double() * norm_reference(z, w[:, None], b[:, None], eps)[0] + e.double() * z).sum()

    args = [t.double() for t in (x, r, w, b)]
    step = 1e-5
    for at, got in enumerate((dx, dres, dw, db)):
        want = torch.empty_like(args[at])
        for i in range(want.numel()):
            moved = [a.clone() for a in args]
            moved[at].view(-1)[i] += step
            up = f(*moved)
            moved[at].view(-1)[i] -= 2 * step
            want.view(-1)[i] = (up - f(*moved)) / (2 * step)
        # fp32 sums of about a hundred terms of size one; differences: rounding 1e-16 * 100 / 1e-5, truncation 1e-10 f'''
        near(got, want, torch.full_like(want, 200 * U * 10 + 1e-8), torch.float32)


def test_lookup_gradient_against_differences():
    """sum(c * lookup(W)) is linear in W: its difference by one table entry, taken through the kernel, is the gradient."""
    g = gen(12)
    V, d, T = 5, 9, 12
    W, c = normal(g, V, d), normal(g, T, d)
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda")
    grad = pkg.embedding_backward(c, tokens, torch.empty_like(W), scale=2.0)
    for v in range(V):
        for j in range(d):
            E = torch.zeros_like(W)
            E[v, j] = 1.0
            f = (c.double() * pkg.embedding_forward(E, tokens, scale=2.0).double()).sum()
            assert abs(f - grad[v, j].double()) <= 2 * (T + 2) * U * c.abs().sum()


def test_layer_norm_of_degenerate_rows():
    """Constant rows (variance 0), a large common level, everything dropped, rows with infinities or NaN: the others are
    untouched by them."""
    g = gen(13)
    for d in (64, 1000, 1024, 5000):
        x = normal(g, 1, 8, d)
        x[0, 1] = 3.0
        x[0, 2] = 1000.0 + x[0, 2]
        x[0, 4, d // 2] = float("nan")
        x[0, 6, 0] = float("inf")
        y, _, mean, rstd = pkg.layer_norm_forward(x, None, None)
        fine = [0, 2, 3, 5, 7]
        assert (y[0, 1] == 0).all() and abs(rstd[0, 1].item() - 1e-5 ** -0.5) < 1e-3
        assert y[0, 4].isnan().all() and y[0, 6].isnan().any() and y[0, fine].isfinite().all()
        check_forward(x[:, fine].contiguous(), None, None, None, 1e-5, 0.0, None, 1,
                      (y[:, fine], x[:, fine], mean[:, fine], rstd[:, fine]), torch.float32)
        y, z, mean, rstd = pkg.layer_norm_forward(torch.full_like(x, float("nan")), None, None, p=1.0, seed=3)
        assert (z == 0).all() and (y == 0).all() and (mean == 0).all()
        zero = torch.zeros_like(mean)
        bad = x[0, :1].clone().expand(8, d).unsqueeze(0).contiguous()
        dres, dx, _, _ = pkg.layer_norm_backward(bad, x.nan_to_num(posinf=0.0), zero, zero + 1, None, p=1.0, seed=3)
        assert (dx == 0).all()


def test_layer_norm_of_views_in_place_and_without_rows():
    """Vectors inside wider buffers at odd places give what dense copies give; outputs over their inputs; parameters in
    slices of X; no rows."""
    g = gen(14)
    for dtype in TYPES:
        for d in (40, 384, 1024, 3000, 20000):
            n, T = 2, 6
            wide = normal(g, n, T, 3 * d + 5, dtype=dtype)
            x, r = wide[..., 1:1 + d], wide[..., 2 + d:2 + 2 * d]
            X = normal(g, n, 2 * d + 3)
            w, b = X[:, 1:1 + d], X[:, 2 + d:2 + 2 * d]
            args = {"residual": r, "p": 0.2, "seed": 6}
            y, z, mean, rstd = pkg.layer_norm_forward(x, w, b, **args)
            dense = pkg.layer_norm_forward(x.contiguous(), w.contiguous(), b.contiguous(), residual=r.contiguous(), p=0.2, seed=6)
            check_forward(x.contiguous(), r.contiguous(), w, b, 1e-5, 0.2, {"seed": 6, "k": 0, "site": 0, "node0": 0}, n, (y, z, mean, rstd), dtype)
            over = wide.clone()
            got = pkg.layer_norm_forward(over[..., 1:1 + d], w, b, residual=over[..., 2 + d:2 + 2 * d], p=0.2, seed=6,
                                         out=over[..., 1:1 + d], z=over[..., 2 + d:2 + 2 * d])
            assert torch.equal(got[0], y) and torch.equal(got[1], z)
            assert torch.equal(over[..., 0], wide[..., 0]) and torch.equal(over[..., 2 + 2 * d:], wide[..., 2 + 2 * d:])
            check_forward(x.contiguous(), r.contiguous(), w.contiguous(), b.contiguous(), 1e-5, 0.2,
                          {"seed": 6, "k": 0, "site": 0, "node0": 0}, n, dense, dtype)

            dy = wide[..., 2 * d + 3:3 * d + 3]
            G = torch.full_like(X, 9.0)
            first = pkg.layer_norm_backward(dy, z, mean, rstd, w, dz=r, p=0.2, seed=6, dweight=G[:, 1:1 + d], dbias=G[:, 2 + d:2 + 2 * d])
            assert (G[:, 0] == 9).all() and (G[:, 1 + d] == 9).all() and (G[:, 2 + 2 * d:] == 9).all()
            dyc, zc = dy.contiguous(), z.clone()
            second = pkg.layer_norm_backward(dyc, zc, mean, rstd, w, dz=r, p=0.2, seed=6, dresidual=dyc, dx=zc)
            scale = first[0].double().abs().max()
            for a, c in zip(first, second):   # the same sums, perhaps in another grouping
                assert (a.double() - c.double()).abs().max() <= (EPS[dtype] + 2 * depth(d) * U) * 4 * max(scale, a.double().abs().max())
    none = torch.empty((2, 0, 16), device="cuda")
    w = torch.ones((2, 16), device="cuda")
    y, _, mean, rstd = pkg.layer_norm_forward(none, w, w)
    dres, _, dw, db = pkg.layer_norm_backward(none, none, mean, rstd, w)
    assert y.shape == none.shape and (dw == 0).all() and (db == 0).all()
    assert pkg.dropout(none, 0.5, 1).shape == none.shape


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(100000, 51), (100000, 77), (3001, 203), (30000, 333), (9001, 701), (80000, 1003), (5001, 1023), (2000, 1501),
                                    (9000, 1999), (2003, 2501), (12000, 3999), (700, 5001), (601, 7001)])
def test_many_dense_rows_of_odd_widths(dtype, rows, d):
    """Rows that are off the alignment each in its own way, more of them than the blocks take at once."""
    test_layer_norm_forward(dtype, 1, rows, d, True, 0.25)
    test_layer_norm_backward(dtype, 1, rows, d, True, 0.25)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [1, 5, 64, 120, 513, 1024, 1030, 2050, 4099, 8185])
def test_vectors_off_the_alignment_alike(dtype, d):
    """Every activation a slice at one place of a buffer of one width: the results are a dense copy's, and nothing beside
    the slices is written."""
    g = gen(17)
    n, T, at = 2, 301, 3
    w, b = 1 + 0.2 * normal(g, n, d), normal(g, n, d)

    def wide(fill=None):
        t = normal(g, n, T, d + 13, dtype=dtype) if fill is None else torch.full((n, T, d + 13), fill, device="cuda", dtype=dtype)
        return t, t[..., at:at + d]

    (_, x), (_, r), (_, dy), (_, e) = wide(), wide(), wide(), wide()
    outs = [wide(9.0) for _ in range(5)]
    mask = {"p": 0.3, "seed": 4, "k": 2, "site": 1}
    y, z, mean, rstd = pkg.layer_norm_forward(x, w, b, residual=r, out=outs[0][1], z=outs[1][1], **mask)
    check_forward(x.contiguous(), r.contiguous(), w, b, 1e-5, 0.3, {**mask, "node0": 0}, n, (y, z, mean, rstd), dtype)
    got = pkg.layer_norm_backward(dy, z, mean, rstd, w, dz=e, dresidual=outs[2][1], dx=outs[3][1], **mask)
    ref = pkg.layer_norm_backward(dy.contiguous(), z.contiguous(), mean, rstd, w, dz=e.contiguous(), **mask)
    size = ref[0].double().abs().max()
    for a, c in zip(got[:2], ref[:2]):   # the same sums, perhaps in another grouping
        assert (a.double() - c.double()).abs().max() <= (EPS[dtype] + 2 * depth(d) * U) * 4 * size
    xh = (z.double() - mean.double()[..., None]) * rstd.double()[..., None]
    near(got[2], (dy.double() * xh).sum(1), (T + 3) * U * (dy.double() * xh).abs().sum(1), torch.float32)
    near(got[3], dy.double().sum(1), T * U * dy.double().abs().sum(1), torch.float32)
    drop = pkg.dropout(x, 0.3, 11, nodes=n, out=outs[4][1])
    assert torch.equal(drop, pkg.dropout(x.contiguous(), 0.3, 11, nodes=n))
    for buf, _ in outs:
        assert (buf[..., :at] == 9).all() and (buf[..., at + d:] == 9).all()


@pytest.mark.parametrize("d", [40, 41, 1030, 4500])
def test_probabilities_that_round_to_zero_and_one(d):
    """p below 2^-17 drops nothing and leaves the factor 1, p above 1 - 2^-17 drops everything, in every operator."""
    g = gen(18)
    x, w = normal(g, 1, 600, d, dtype=torch.bfloat16), torch.ones(d, device="cuda")
    for p in (1e-6, 1 - 1e-6):
        keep = torch.ones_like(x) if p < 0.5 else torch.zeros_like(x)
        assert torch.equal(pkg.dropout(x, p, 5), x * keep)
        y, z, mean, rstd = pkg.layer_norm_forward(x, w, None, p=p, seed=5)
        assert torch.equal(z, x * keep)
        dres, dx, _, _ = pkg.layer_norm_backward(x, z, mean, rstd, w, p=p, seed=5)
        assert torch.equal(dx, dres * keep) and (p > 0.5 or dres.abs().max() > 0)


@pytest.mark.parametrize("d", [96, 97, 1000, 9000])
def test_parameters_shared_and_left_out(d):
    """One weight and one table for all nodes (node stride 0), a weight without a bias, no weight at all."""
    g = gen(19)
    n, T, V = 3, 7, 11
    x, w, b = normal(g, n, T, d), 1 + 0.2 * normal(g, d), normal(g, d)
    shared = pkg.layer_norm_forward(x, w.expand(n, d), b.expand(n, d))
    alone = pkg.layer_norm_forward(x, w, b)
    assert all(torch.equal(a, c) for a, c in zip(shared[::2], alone[::2]))
    y, _, mean, rstd = pkg.layer_norm_forward(x, w, None)
    check_forward(x, None, w[None], None, 1e-5, 0.0, None, 1, (y.view(1, n * T, d), x.view(1, n * T, d), mean, rstd), torch.float32)
    bare = pkg.layer_norm_forward(x, None, None)
    check_forward(x, None, None, None, 1e-5, 0.0, None, 1, (bare[0].view(1, n * T, d), x.view(1, n * T, d), mean, rstd), torch.float32)
    dy = normal(g, n, T, d)
    per_node = pkg.layer_norm_backward(dy, x, mean, rstd, w.expand(n, d))
    total = pkg.layer_norm_backward(dy, x, mean, rstd, w)
    assert per_node[2].shape == (n, d)
    for a, c, terms in ((per_node[2], total[2], dy * (x - mean[..., None]) * rstd[..., None]), (per_node[3], total[3], dy)):
        assert ((a.double().sum(0) - c.double()).abs() <= 2 * (n * T + 3) * U * terms.double().abs().sum((0, 1))).all()
    none = pkg.layer_norm_backward(dy, x, mean, rstd, None)
    ones = pkg.layer_norm_backward(dy, x, mean, rstd, torch.ones(d, device="cuda"))
    assert torch.equal(none[0], ones[0]) and none[2] is None and none[3] is None
    table = normal(g, V, d)
    tokens = torch.randint(0, V, (n, T), generator=g, device="cuda")
    assert torch.equal(pkg.embedding_forward(table.expand(n, V, d), tokens), table[tokens])


def test_activations_beyond_32_bit_offsets():
    """Vectors 2^27 elements apart: 20 of them span 2.6e9 elements."""
    wide = torch.zeros((20, 2 ** 27), dtype=torch.bfloat16, device="cuda")
    x = wide[:, 8:8 + 512]
    x.copy_(normal(gen(15), 20, 512))
    dense = x.contiguous()
    w, b = torch.full((512,), 1.5, device="cuda"), torch.full((512,), 0.25, device="cuda")
    y, _, mean, rstd = pkg.layer_norm_forward(x, w, b)
    want = pkg.layer_norm_forward(dense, w, b)
    assert torch.equal(y, want[0]) and torch.equal(mean, want[2])
    assert torch.equal(pkg.dropout(x, 0.3, 4), pkg.dropout(dense, 0.3, 4))
    got = pkg.layer_norm_backward(x, x, mean, rstd, w)
    ref = pkg.layer_norm_backward(dense, dense, mean, rstd, w)
    assert all(torch.equal(a, c) for a, c in zip(got, ref))


# ---- streams, capture, refusals --------------------------------------------------------------------
def test_other_streams_and_graph_capture():
    g = gen(16)
    x, r, w, b = norm_inputs(g, 2, 64, 512, torch.bfloat16)
    tokens = torch.randint(0, 300, (2, 64), generator=g, device="cuda")
    table = normal(g, 2, 300, 512)
    grad = torch.empty_like(table)

    def block(stream=None):
        e = pkg.embedding_forward(table, tokens, dtype=torch.bfloat16, stream=stream)
        y, z, mean, rstd = pkg.layer_norm_forward(e, w, b, residual=r, p=0.1, seed=1, stream=stream)
        dres, dx, dw, db = pkg.layer_norm_backward(y, z, mean, rstd, w, p=0.1, seed=1, stream=stream)
        out = pkg.dropout(dx, 0.2, 3, nodes=2, stream=stream)
        return [e, y, z, mean, rstd, dres, dx, dw, db, out, pkg.embedding_backward(out, tokens, grad, stream=stream)]

    want = [t.clone() for t in block()]
    grad.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = block(stream=s)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    torch.cuda.current_stream().wait_stream(s)
    grad.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))


def test_refusals():
    x = torch.ones((2, 4, 16), device="cuda")
    w = torch.ones((2, 16), device="cuda")
    tokens = torch.zeros((2, 4), dtype=torch.int64, device="cuda")
    table = torch.ones((2, 5, 16), device="cuda")
    mean = torch.zeros((2, 4), device="cuda")
    calls = [
        lambda: pkg.embedding_forward(table.half(), tokens),
        lambda: pkg.embedding_forward(table, tokens.float()),
        lambda: pkg.embedding_forward(table, tokens[:1]),
        lambda: pkg.embedding_forward(table, tokens, out=torch.empty((2, 4, 15), device="cuda")),
        lambda: pkg.embedding_forward(table, tokens, dtype=torch.float64),
        lambda: pkg.embedding_forward(table.transpose(1, 2), tokens),
        lambda: pkg.embedding_forward(table.cpu(), tokens.cpu()),
        lambda: pkg.embedding_backward(x[..., :15], tokens, table),
        lambda: pkg.embedding_backward(x[:1].expand(2, 4, 16).repeat(1, 200, 1), tokens.repeat(1, 200), table,
                                       scratch=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: pkg.embedding_backward(x, tokens, torch.ones((1, 5, 16), device="cuda").expand(2, 5, 16)),
        lambda: pkg.dropout(x, 1.5, 0),
        lambda: pkg.dropout(x, float("nan"), 0),
        lambda: pkg.dropout(x, 0.5, 0, nodes=3),
        lambda: pkg.dropout(x, 0.5, 0, k=-1),
        lambda: pkg.dropout(x, 0.5, 0, site=2 ** 30),
        lambda: pkg.dropout(x, 0.5, 0, out=x.half()),
        lambda: pkg.dropout(x.double(), 0.5, 0),
        lambda: pkg.dropout(x.transpose(1, 2), 0.5, 0),
        lambda: pkg.layer_norm_forward(x, w[:, :8], w),
        lambda: pkg.layer_norm_forward(x, w, w, eps=-1.0),
        lambda: pkg.layer_norm_forward(x, w, w, residual=x[:1]),
        lambda: pkg.layer_norm_forward(x, w, w.half()),
        lambda: pkg.layer_norm_forward(x, w, w, mean=mean.double()),
        lambda: pkg.layer_norm_backward(x, x, mean, mean, w, dx=x),
        lambda: pkg.layer_norm_backward(x, x, mean[:1], mean, w),
        lambda: pkg.layer_norm_backward(x, x, mean, mean, w, accumulate=True),
        lambda: pkg.layer_norm_backward(x.half(), x, mean, mean, w),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(pkg.GpgaError) as err:
            call()
        assert err.value.status == pkg.GPGA_ERR_INVALID_ARG and str(err.value), i
