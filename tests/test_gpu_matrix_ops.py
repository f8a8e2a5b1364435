"""The gated feed-forward block and its gradient on the GPU, against plain forms in 64 bits.

Two kinds of inputs.  Small whole numbers with relu: every sum is exact in fp32 whatever its order, so the results have to be
equal, bit for bit, at every size and layout.  Normal numbers: the error of every element is held to a bound from the
roundings on its way, derived in `block_bound` before any run:

  U            half a step of the activations' type: what one rounding is off by, relative to the value
  sums         16-bit operands: K / 16 matrix instructions, each of which cuts at most a step (2^-23) of the running sum off, plus up to 70
               partial sums; fp32 operands: 4.4 such cuts per 64 columns of the chunk's own sum, K / 64 sums of chunks (2^-24
               each), 2^-21 for products of pieces that are left out, 40 for the reduction of a call of few tokens
  fp32 weights beside 16-bit activations: two values, 2^-16 (bfloat16) or 2^-22 and 2^-25 absolute (fp16) off
"""
import math

import pytest
import torch

import paper_2105_09080_b200 as pkg

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -134, F16: 2.0 ** -25}
KINDS = ["silu", "gelu", "relu"]
ACT = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}
# one token to many, every path (few tokens; one block, clusters, pairs of blocks), sizes around the tiles' and vectors' edges
SIZES = [(1, 1, 1, 1), (1, 1, 7, 5), (2, 3, 16, 24), (1, 8, 129, 333), (1, 9, 64, 64), (2, 17, 130, 70), (1, 32, 257, 129), (1, 33, 128, 128),
         (3, 40, 100, 36), (2, 64, 72, 200), (1, 127, 65, 63), (1, 128, 256, 128), (1, 129, 8, 264), (2, 255, 515, 77), (1, 300, 1373, 129),
         (1, 700, 520, 1030), (1, 2500, 64, 96), (5, 260, 300, 310), (1, 4500, 264, 520)]
TYPES = [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)]


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def whole(shape, gen, dtype, some=0.25):
    """-1, 0 or 1, mostly 0."""
    r = torch.rand(shape, generator=gen, device="cuda")
    return ((r < some / 2).float() - (r > 1 - some / 2).float()).to(dtype)


def whole_inputs(n, t, d, f, dtype, wtype, seed=0):
    g = generator(seed)
    return whole((n, t, d), g, dtype), whole((n, f, d), g, wtype), whole((n, f, d), g, wtype), whole((n, d, f), g, wtype)


def whole_forward(x, gate, up, down):
    """What the block has to give, exactly, for whole numbers and relu: values are rounded where they are stored."""
    dtype = x.dtype
    x, gate, up, down = (v.double() for v in (x, gate, up, down))
    g, u = x @ gate.mT, x @ up.mT
    h = (torch.relu(g) * u).to(dtype).double()
    return (h @ down.mT).to(dtype), g.to(dtype), u.to(dtype)


def whole_backward(dy, x, g, u, gate, up, down):
    dtype = x.dtype
    dy, x, g, u, gate, up, down = (v.double() for v in (dy, x, g, u, gate, up, down))
    dh, on = dy @ down, (g > 0).double()
    h, du, dg = ((v).to(dtype).double() for v in (g * on * u, dh * g * on, dh * u * on))
    return (dg @ gate + du @ up).to(dtype), dg.mT @ x, du.mT @ x, dy.mT @ h


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype,wtype", TYPES, ids=str)
def test_forward_of_whole_numbers_is_exact(size, dtype, wtype):
    x, gate, up, down = whole_inputs(*size, dtype, wtype)
    want = whole_forward(x, gate, up, down)
    got = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    for name, a, b in zip("ygu", got, want):
        assert a.dtype is dtype and torch.equal(a, b), name
    y, none_g, none_u = pkg.feed_forward_forward(x, gate, up, down, activation="relu", keep=False)
    assert none_g is None and none_u is None and torch.equal(y, want[0])
    pkg.token_status()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype,wtype", TYPES, ids=str)
def test_backward_of_whole_numbers_is_exact(size, dtype, wtype):
    n, t, d, f = size
    x, gate, up, down = whole_inputs(n, t, d, f, dtype, wtype, seed=1)
    g = generator(2)
    dy = whole((n, t, d), g, dtype)
    gv, uv = ((3 * torch.rand((n, t, f), generator=g, device="cuda")).floor() - 1 for _ in range(2))
    gv, uv = gv.to(dtype), uv.to(dtype)
    want = whole_backward(dy, x, gv, uv, gate, up, down)
    got = pkg.feed_forward_backward(dy, x, gv, uv, gate, up, down, activation="relu")
    for name, a, b in zip(("dx", "dgate", "dup", "ddown"), got, want):
        assert a.dtype is (dtype if name == "dx" else wtype) and torch.equal(a, b.to(a.dtype)), name
    pkg.token_status()


def normal(shape, gen, dtype, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen).to(dtype)


def normal_inputs(n, t, d, f, dtype, wtype, seed):
    g = generator(seed)
    return (normal((n, t, d), g, dtype), normal((n, f, d), g, wtype, d ** -0.5), normal((n, f, d), g, wtype, d ** -0.5),
            normal((n, d, f), g, wtype, f ** -0.5))


def sums(k, dtype):
    return 2.0 ** -21 + (40 + k / 64) * 2.0 ** -23 if dtype is F32 else (k / 16 + 70) * 2.0 ** -23


def weight_error(w, dtype):
    if dtype is F32 or w.dtype is not F32:
        return torch.zeros_like(w, dtype=torch.float64)
    return w.double().abs() * (2.0 ** -16 if dtype is BF16 else 2.0 ** -22) + (2.0 ** -25 if dtype is F16 else 0.0)


def block_bound(x, gate, up, down, kind):
    """(y, g, u) in 64 bits and how far each of their elements may be off."""
    dtype, X, A, B, D = x.dtype, *(v.double() for v in (x, gate, up, down))
    g, u = X @ A.mT, X @ B.mT
    eg, eu = (X.abs() @ (w.double().abs() * sums(X.shape[-1], dtype) + weight_error(w, dtype)).mT for w in (gate, up))
    a = ACT[kind](g)
    h = a * u
    # |act'| <= 1.13; the activation itself: 2^-18 (16-bit) or 2^-21 of the value, and of v where 1 + erf cancels
    own = (2.0 ** -18 if dtype is not F32 else 2.0 ** -21) * (h.abs() + (g * u).abs())
    eh = 1.13 * eg * (u.abs() + eu) + a.abs() * eu + own
    if dtype is not F32:
        eh = eh + U[dtype] * (h.abs() + eh) + TINY[dtype]
    y = h @ D.mT
    ey = eh @ D.abs().mT + (h.abs() + eh) @ (D.abs() * sums(h.shape[-1], dtype) + weight_error(down, dtype)).mT
    return [(v, e + U[dtype] * (v.abs() + e) + TINY[dtype]) for v, e in ((y, ey), (g, eg), (u, eu))]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (2, 5, 77, 130), (1, 24, 512, 700), (2, 90, 129, 333), (1, 300, 1024, 260), (1, 600, 64, 1500)], ids=str)
@pytest.mark.parametrize("dtype,wtype", TYPES, ids=str)
def test_forward_against_64_bits(kind, size, dtype, wtype):
    args = normal_inputs(*size, dtype, wtype, seed=3)
    for got, (want, bound) in zip(pkg.feed_forward_forward(*args, activation=kind), block_bound(*args, kind)):
        assert ((got.double() - want).abs() <= bound).all()


def slope(g, kind):
    g = g.detach().clone().requires_grad_()
    with torch.enable_grad():
        s, = torch.autograd.grad(ACT[kind](g).sum(), g)
    return s


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (2, 5, 77, 130), (2, 90, 129, 333), (1, 300, 520, 260), (1, 1500, 64, 200)], ids=str)
@pytest.mark.parametrize("dtype,wtype", TYPES, ids=str)
def test_backward_against_64_bits(kind, size, dtype, wtype):
    n, t, d, f = size
    x, gate, up, down = normal_inputs(*size, dtype, wtype, seed=4)
    gen = generator(5)
    dy, g, u = normal((n, t, d), gen, dtype), normal((n, t, f), gen, dtype, 1.5), normal((n, t, f), gen, dtype)
    X, DY, G, V, A, B, D = (v.double() for v in (x, dy, g, u, gate, up, down))
    a, s = ACT[kind](G), slope(G, kind)
    dh = DY @ D
    eh = DY.abs() @ (D.abs() * sums(d, dtype) + weight_error(down, dtype))
    fa = 2.0 ** -18 if dtype is not F32 else 2.0 ** -21
    parts = {}
    for name, value, factor, own in (("h", a * V, None, (a * V).abs() + (G * V).abs()), ("du", dh * a, a, dh.abs() * (a.abs() + G.abs())),
                                     ("dg", dh * V * s, V * s, (dh * V).abs() * (1.2 + G.abs()))):
        e = fa * own + (eh * factor.abs() if factor is not None else 0.0)
        if dtype is not F32:
            e = e + U[dtype] * (value.abs() + e) + TINY[dtype]
        parts[name] = value, e
    (h, e_h), (du, e_du), (dg, e_dg) = parts["h"], parts["du"], parts["dg"]
    dx = dg @ A + du @ B
    e_dx = sum((v.abs() + e) @ (w.double().abs() * sums(2 * f, dtype) + weight_error(w, dtype)) + e @ w.double().abs()
               for v, e, w in ((dg, e_dg, gate), (du, e_du, up)))
    want = [(dx, e_dx)]
    for v, e, o in ((dg, e_dg, X), (du, e_du, X)):
        want.append((v.mT @ o, e.mT @ o.abs() + sums(t, dtype) * ((v.abs() + e).mT @ o.abs())))
    want.append((DY.mT @ h, DY.abs().mT @ e_h + sums(t, dtype) * (DY.abs().mT @ (h.abs() + e_h))))
    for got, (value, e) in zip(pkg.feed_forward_backward(dy, x, g, u, gate, up, down, activation=kind), want):
        bound = e + U[got.dtype] * (value.abs() + e) + TINY[got.dtype]
        assert ((got.double() - value).abs() <= bound).all()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gradient_against_differences(kind):
    """Along a direction v of all inputs: sum(w y) at two points 2 h apart.  Its own error: the rounding of y there (bounded
    by block_bound) over 2 h, and the curvature, at most h^2 of the third difference, measured with a second h."""
    n, t, d, f = 2, 40, 36, 52
    args = normal_inputs(n, t, d, f, F32, F32, seed=6)
    gen = generator(7)
    way = [normal(a.shape, gen, F32) * a.abs().mean() for a in args]
    w = normal((n, t, d), gen, F32)
    y, g, u = pkg.feed_forward_forward(*args, activation=kind)
    grads = pkg.feed_forward_backward(w, args[0], g, u, *args[1:], activation=kind)
    along = sum((a.double() * b.double()).sum() for a, b in zip(grads, way))

    def difference(h):
        ends, noise = [], 0.0
        for s in (h, -h):
            at = [a + s * v for a, v in zip(args, way)]
            ends.append((w.double() * pkg.feed_forward_forward(*at, activation=kind)[0].double()).sum())
            noise += float((w.double().abs() * block_bound(*at, kind)[0][1]).sum())
        return (ends[0] - ends[1]) / (2 * h), noise / (2 * h)

    (a, na), (b, nb) = difference(2.0 ** -5), difference(2.0 ** -6)
    # the difference quotient is along + c h^2 + ...: the two give c, and twice its share is allowed
    curvature = 2 * abs(float(a - b)) / 3 + na + nb
    size = sum(float((p.double().abs() * q.double().abs()).sum()) for p, q in zip(grads, way))
    assert abs(float(along - b)) <= curvature + nb + 2.0 ** -18 * size
    assert curvature <= 0.02 * abs(float(along)) + 0.02 * size      # or the test says nothing


def strided(value, pad, lead=0):
    """The same values in rows `pad` elements further apart, `lead` elements into a buffer; the rest is NaN."""
    n, r, c = value.shape
    buf = torch.full((n * r * (c + pad) + lead + 8,), float("nan"), dtype=value.dtype, device="cuda")
    view = buf[lead:lead + n * r * (c + pad)].view(n, r, c + pad)[..., :c]
    view.copy_(value)
    return view, buf


@pytest.mark.parametrize("pad,lead", [(8, 0), (3, 0), (5, 1), (0, 1), (16, 8)])
@pytest.mark.parametrize("size", [(2, 5, 77, 130), (2, 40, 72, 136), (1, 300, 128, 515)], ids=str)
@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (BF16, BF16), (F16, F32)], ids=str)
def test_rows_apart_and_off_the_alignment(size, dtype, wtype, pad, lead):
    """Inputs and outputs anywhere: the same results, and nothing written between the rows."""
    x, gate, up, down = whole_inputs(*size, dtype, wtype, seed=8)
    y, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    grads = pkg.feed_forward_backward(x, x, g, u, gate, up, down, activation="relu")
    wide = [strided(v, pad, lead)[0] for v in (x, gate, up, down)]
    outs = [strided(v, pad, lead) for v in (y, g, u)]
    pkg.feed_forward_forward(*wide, activation="relu", out=outs[0][0], g=outs[1][0], u=outs[2][0])
    for (view, buf), value in zip(outs, (y, g, u)):
        assert torch.equal(view, value) and (~buf.isnan()).sum() == value.numel()
    outs = [strided(torch.zeros_like(v), pad, lead) for v in grads]
    pkg.feed_forward_backward(wide[0], wide[0], strided(g, pad, lead)[0], strided(u, pad, lead)[0], *wide[1:], activation="relu", dx=outs[0][0],
                              dgate=outs[1][0], dup=outs[2][0], ddown=outs[3][0])
    for (view, buf), value in zip(outs, grads):
        assert torch.equal(view, value) and (~buf.isnan()).sum() == value.numel()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_slices_of_the_state_matrix(dtype):
    """Weights in the rows of X, gradients into the same places of G, added to what is there."""
    n, t, d, f = 3, 70, 24, 40
    s, lead = f * d, 5
    gen = generator(9)
    X, G = (whole((n, lead + 3 * s + 7), gen, F32) for _ in range(2))

    def parts(M):
        shapes = ((f, d), (f, d), (d, f))
        return [M[:, lead + i * s:lead + (i + 1) * s].unflatten(1, shape) for i, shape in enumerate(shapes)]

    x, dy = whole((n, t, d), gen, dtype), whole((n, t, d), gen, dtype)
    y, g, u = pkg.feed_forward_forward(x, *parts(X), activation="relu")
    want = whole_forward(x, *parts(X))
    assert all(torch.equal(a, b) for a, b in zip((y, g, u), want))
    before = G.clone()
    dgate, dup, ddown = parts(G)
    dx, *_ = pkg.feed_forward_backward(dy, x, g, u, *parts(X), activation="relu", dgate=dgate, dup=dup, ddown=ddown, accumulate=True)
    ref = whole_backward(dy, x, g, u, *parts(X))
    assert torch.equal(dx, ref[0])
    for got, old, add in zip(parts(G), parts(before), ref[1:]):
        assert torch.equal(got.double(), old.double() + add)
    assert torch.equal(G[:, :lead], before[:, :lead]) and torch.equal(G[:, lead + 3 * s:], before[:, lead + 3 * s:])


@pytest.mark.parametrize("size", [(2, 30, 24, 40), (1, 300, 129, 77)], ids=str)
def test_16_bit_gradients_added_to(size):
    """Sums of whole numbers below 2^11 (fp16): the sum of old and new is rounded once."""
    n, t, d, f = size
    x, gate, up, down = whole_inputs(*size, F16, F16, seed=18)
    gen = generator(19)
    y, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    grads = pkg.feed_forward_backward(x, x, g, u, gate, up, down, activation="relu")[1:]
    old = [whole(w.shape, gen, F16) for w in grads]
    new = [w.clone() for w in old]
    pkg.feed_forward_backward(x, x, g, u, gate, up, down, activation="relu", dgate=new[0], dup=new[1], ddown=new[2], accumulate=True)
    exact = whole_backward(x, x, g, u, gate, up, down)[1:]
    assert all(torch.equal(a, (b.double() + c).to(F16)) for a, b, c in zip(new, old, exact))


@pytest.mark.parametrize("rows", [3, 20, 200])
def test_outputs_in_the_place_of_inputs(rows):
    x, gate, up, down = whole_inputs(2, rows, 40, 56, BF16, BF16, seed=10)
    y, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    over = x.clone()
    assert pkg.feed_forward_forward(over, gate, up, down, activation="relu", out=over)[0] is over and torch.equal(over, y)
    dy = whole((2, rows, 40), generator(11), BF16)
    dx, *rest = pkg.feed_forward_backward(dy, x, g, u, gate, up, down, activation="relu")
    for which in (0, 1):
        a = [dy.clone(), x.clone()]
        got, *others = pkg.feed_forward_backward(*a, g, u, gate, up, down, activation="relu", dx=a[which])
        assert got is a[which] and torch.equal(got, dx) and all(torch.equal(p, q) for p, q in zip(others, rest))


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("rows", [6, 31, 300])
def test_a_bad_token_stays_alone(dtype, rows):
    """NaN and infinities of one token reach that token's outputs only (and the weights' gradients)."""
    x, gate, up, down = normal_inputs(1, rows, 64, 80, dtype, dtype, seed=12)
    clean = pkg.feed_forward_forward(x, gate, up, down)
    dclean = pkg.feed_forward_backward(x, x, clean[1], clean[2], gate, up, down)[0]
    for bad in (float("nan"), float("inf")):
        z = x.clone()
        z[0, 4, 3] = bad
        got = pkg.feed_forward_forward(z, gate, up, down)
        dx = pkg.feed_forward_backward(z, x, clean[1], clean[2], gate, up, down)[0]
        others = [i for i in range(rows) if i != 4]
        for a, b in zip((*got, dx), (*clean, dclean)):
            assert torch.equal(a[:, others], b[:, others])
            assert not a[0, 4].isfinite().all()


LARGE = [(1, 3000, 1030, 1100), (3, 1501, 700, 780)]      # fp32 as pairs of fp16 values


@pytest.mark.parametrize("size", LARGE, ids=str)
def test_large_fp32_products_of_whole_numbers(size):
    """Powers of two before and after the products change nothing: still exact, off the alignment too, and added to."""
    x, gate, up, down = whole_inputs(*size, F32, F32, seed=20)
    dy = whole(x.shape, generator(21), F32)
    want = whole_forward(x, gate, up, down)
    got = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(pkg.feed_forward_forward(x, gate, up, down, activation="relu", keep=False)[0], want[0])
    ref = whole_backward(dy, x, got[1], got[2], gate, up, down)
    grads = pkg.feed_forward_backward(dy, x, got[1], got[2], gate, up, down, activation="relu")
    assert all(torch.equal(a, b.float()) for a, b in zip(grads, ref))
    wide = [strided(v, 3, 1)[0] for v in (x, gate, up, down)]
    outs = [strided(v, 3, 1) for v in want]
    pkg.feed_forward_forward(*wide, activation="relu", out=outs[0][0], g=outs[1][0], u=outs[2][0])
    assert all(torch.equal(view, v) and (~buf.isnan()).sum() == v.numel() for (view, buf), v in zip(outs, want))
    new = [torch.ones_like(w) for w in (gate, up, down)]
    pkg.feed_forward_backward(dy, wide[0], outs[1][0], outs[2][0], *wide[1:], activation="relu", dgate=new[0], dup=new[1], ddown=new[2], accumulate=True)
    assert all(torch.equal(a, (1 + b).float()) for a, b in zip(new, ref[1:]))
    assert all(torch.equal(a, b) for a, b in zip(pkg.feed_forward_backward(dy, x, got[1], got[2], gate, up, down, activation="relu"), grads))


@pytest.mark.parametrize("spread", [0, 12])
def test_large_fp32_products_against_64_bits(spread):
    """Tokens whose sizes differ by 2^12: every element within the bound of its own row.  Two fp16 values hold 24 bits of what
    is at least 2^-17 of an array's largest value, and 2^-40 of that below; the largest of some million normal numbers is
    below 8, so a value 2^-12 times a normal one keeps 2^-24 beside 2^-37 absolute, which the bound's 40 steps of the row's own sums cover
    where those are above 2^-14: with 1030 terms of 2^-12 they are."""
    x, gate, up, down = normal_inputs(1, 3000, 1030, 1100, F32, F32, seed=22)
    x = x * torch.exp2(-torch.arange(3000, device="cuda") % (spread + 1)).float()[None, :, None]
    for kind in ("silu", "gelu"):
        for got, (want, bound) in zip(pkg.feed_forward_forward(x, gate, up, down, activation=kind)[1:], block_bound(x, gate, up, down, kind)[1:]):
            assert ((got.double() - want).abs() <= bound).all()
    if spread == 0:
        (want, bound), *_ = block_bound(x, gate, up, down, "silu")
        assert ((pkg.feed_forward_forward(x, gate, up, down)[0].double() - want).abs() <= bound).all()


def test_large_fp32_products_leave_bad_tokens_alone():
    x, gate, up, down = normal_inputs(1, 3000, 1030, 1100, F32, F32, seed=23)
    clean = pkg.feed_forward_forward(x, gate, up, down)
    dclean = pkg.feed_forward_backward(x, x, clean[1], clean[2], gate, up, down)[0]
    z = x.clone()
    z[0, 4, 3], z[0, 2900, 1000] = float("inf"), float("nan")
    got = pkg.feed_forward_forward(z, gate, up, down)
    dx = pkg.feed_forward_backward(z, x, clean[1], clean[2], gate, up, down)[0]
    others = [i for i in range(3000) if i not in (4, 2900)]
    # the largest finite value may be another one than before, so the powers of two may differ, and with them the last bits
    for a, b in zip((*got, dx), (*clean, dclean)):
        assert (a[:, others] - b[:, others]).abs().max() <= 2.0 ** -18 * b.abs().max()
        assert not a[0, 4].isfinite().all() and not a[0, 2900].isfinite().all()
    zero = pkg.feed_forward_forward(x * 0, gate, up, down)
    assert all((v == 0).all() for v in zero)


@pytest.mark.parametrize("factor", [2.0 ** 60, 2.0 ** -60, 2.0 ** 100])
def test_large_fp32_products_of_extreme_numbers(factor):
    """Powers of two on inputs pass through g and u exactly, far from one too."""
    x, gate, up, down = normal_inputs(1, 3000, 1030, 1100, F32, F32, seed=24)
    _, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    _, g2, u2 = pkg.feed_forward_forward(x * factor, gate, up, down, activation="relu")
    assert torch.equal(g2, g * factor) and torch.equal(u2, u * factor)


def test_no_tokens():
    gate, up, down = (torch.ones(s, device="cuda", dtype=BF16) for s in ((2, 12, 8), (2, 12, 8), (2, 8, 12)))
    x = torch.empty((2, 0, 8), device="cuda", dtype=BF16)
    y, g, u = pkg.feed_forward_forward(x, gate, up, down)
    assert y.shape == (2, 0, 8) and g.shape == (2, 0, 12)
    for given in (None, F32):
        outs = {} if given is None else {k: torch.full_like(w, 7.0, dtype=F32) for k, w in (("dgate", gate), ("dup", up), ("ddown", down))}
        dx, *grads = pkg.feed_forward_backward(x, x, g, u, gate, up, down, **outs)
        assert dx.shape == (2, 0, 8) and all((w == 0).all() for w in grads)
        if outs:
            outs = {k: torch.full_like(w, 7.0) for k, w in outs.items()}
            pkg.feed_forward_backward(x, x, g, u, gate, up, down, accumulate=True, **outs)
            assert all((w == 7).all() for w in outs.values())


@pytest.mark.parametrize("size", [(2, 7, 64, 96), (3, 100, 130, 70), (1, 600, 320, 512)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_same_bits_every_time_on_streams_and_in_graphs(size, dtype):
    """Twice the same; on another stream; two streams at once; captured and replayed with other inputs, an eager call of the
    same tensors before and after."""
    args = normal_inputs(*size, dtype, dtype, seed=13)
    other = normal_inputs(*size, dtype, dtype, seed=14)

    def run(a):
        y, g, u = pkg.feed_forward_forward(*a)
        return (y, g, u, *pkg.feed_forward_backward(y, a[0], g, u, *a[1:]))

    want, want_other = run(args), run(other)
    assert all(torch.equal(a, b) for a, b in zip(run(args), want))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s, a in zip(streams, (args, other)):
        with torch.cuda.stream(s):
            got.append(run(a))
    y = pkg.feed_forward_forward(*args, stream=streams[0])[0]
    torch.cuda.synchronize()
    assert torch.equal(y, want[0])
    for r, w in zip(got, (want, want_other)):
        assert all(torch.equal(a, b) for a, b in zip(r, w))
    held = [a.clone() for a in args]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(run(held))
    for h, o in zip(held, other):
        h.copy_(o)
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for r in outs:
        assert all(torch.equal(a, b) for a, b in zip(r, want_other))
    assert all(torch.equal(a, b) for a, b in zip(run(args), want))


def test_given_scratch_is_used_and_checked():
    x, gate, up, down = whole_inputs(1, 200, 64, 96, F32, F32, seed=15)
    want = pkg.feed_forward_forward(x, gate, up, down, activation="relu")[0]
    scratch = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    assert torch.equal(pkg.feed_forward_forward(x, gate, up, down, activation="relu", scratch=scratch)[0], want)
    with pytest.raises(pkg.GpgaError):
        pkg.feed_forward_forward(x, gate, up, down, scratch=scratch[:1024])


def test_refusals_of_the_binding():
    x, gate, up, down = whole_inputs(2, 10, 16, 24, BF16, BF16)
    y, g, u = pkg.feed_forward_forward(x, gate, up, down)
    wrong = [
        lambda: pkg.feed_forward_forward(x.double(), gate, up, down),
        lambda: pkg.feed_forward_forward(x, gate.half(), up, down),
        lambda: pkg.feed_forward_forward(x, gate, up.float(), down),
        lambda: pkg.feed_forward_forward(x, gate, up, down.mT),
        lambda: pkg.feed_forward_forward(x, gate, up[:, :20], down),
        lambda: pkg.feed_forward_forward(x[..., :8], gate, up, down),
        lambda: pkg.feed_forward_forward(x[:, :3], gate, up, down[:1]),
        lambda: pkg.feed_forward_forward(x, gate, up, down, activation="tanh"),
        lambda: pkg.feed_forward_forward(x, gate, up, down, keep=False, g=g, u=u),
        lambda: pkg.feed_forward_forward(x, gate, up, down, out=y.float()),
        lambda: pkg.feed_forward_forward(x, gate, up, down, g=g[..., :20]),
        lambda: pkg.feed_forward_forward(x.float(), gate, up, down),
        lambda: pkg.feed_forward_forward(x, gate[:, :0], up[:, :0], down[..., :0]),
        lambda: pkg.feed_forward_backward(x, x, g, u, gate, up, down, accumulate=True),
        lambda: pkg.feed_forward_backward(x, x, g, u, gate, up, down, dgate=torch.empty_like(gate, dtype=F16)),
        lambda: pkg.feed_forward_backward(x, x, g, u, gate, up, down, dgate=torch.empty_like(gate, dtype=F32), dup=torch.empty_like(up)),
        lambda: pkg.feed_forward_backward(x, x, g, u, gate, up, down, dgate=gate[:1].expand(2, 24, 16)),
        lambda: pkg.feed_forward_backward(x, x, g[:, :5], u, gate, up, down),
        lambda: pkg.feed_forward_backward(x.float(), x, g, u, gate, up, down),
    ]
    for call in wrong:
        with pytest.raises(pkg.GpgaError):
            call()
    torch.cuda.synchronize()


def test_shared_weights_of_all_nodes():
    """One matrix for all nodes (node stride 0): read, never written."""
    x, gate, up, down = whole_inputs(3, 50, 32, 40, BF16, BF16, seed=16)
    one = [w[:1].expand_as(w) for w in (gate, up, down)]
    got = pkg.feed_forward_forward(x, *one, activation="relu")
    assert all(torch.equal(a, b) for a, b in zip(got, whole_forward(x, *(w.contiguous() for w in one))))
    few = pkg.feed_forward_forward(x[:, :5].contiguous(), *one, activation="relu")[0]
    assert torch.equal(few, got[0][:, :5])


def test_offsets_past_32_bits():
    """Weights of the second node more than 2^32 elements behind the first's; tokens whose kept rows lie past 2^31 elements."""
    gen = generator(17)
    d, f = 16, 24
    X = torch.empty((2, 2 ** 31 + 2 ** 20 + 3 * f * d), dtype=BF16, device="cuda")
    small = [whole(s, gen, BF16) for s in ((2, f, d), (2, f, d), (2, d, f))]
    views = [X[:, -(i + 1) * f * d:X.shape[1] - i * f * d].unflatten(1, s.shape[1:]) for i, s in enumerate(small)]
    for v, s in zip(views, small):
        v.copy_(s)
    for rows in (4, 150):
        x = whole((2, rows, d), gen, BF16)
        for a, b in zip(pkg.feed_forward_forward(x, *views, activation="relu"), pkg.feed_forward_forward(x, *small, activation="relu")):
            assert torch.equal(a, b)
    del X, views
    rows, f = 2 ** 20 + 77, 2056
    x, gate, up, down = (whole(s, gen, BF16, 0.5) for s in ((1, rows, d), (1, f, d), (1, f, d), (1, d, f)))
    assert rows * f > 2 ** 31
    y, g, u = pkg.feed_forward_forward(x, gate, up, down, activation="relu")
    for part in (slice(0, 200), slice(rows - 300, rows)):
        want = whole_forward(x[:, part], gate, up, down)
        assert all(torch.equal(a[:, part], b) for a, b in zip((y, g, u), want))
    dx = pkg.feed_forward_backward(y, x, g, u, gate, up, down, activation="relu")[0]
    part = slice(rows - 300, rows)
    assert torch.equal(dx[:, part], whole_backward(y[:, part], x[:, part], g[:, part], u[:, part], gate, up, down)[0])


def test_a_wait_that_runs_out_is_reported_once():
    pkg.token_status()
    assert pkg.lib().gpga_selftest_token_wait(None) == pkg.GPGA_OK
    with pytest.raises(pkg.GpgaError) as err:
        pkg.token_status()
    assert err.value.status == pkg.GPGA_ERR_TIMEOUT
    pkg.token_status()
    x, gate, up, down = whole_inputs(1, 100, 32, 40, F32, F32)
    assert torch.equal(pkg.feed_forward_forward(x, gate, up, down, activation="relu")[0], whole_forward(x, gate, up, down)[0])
