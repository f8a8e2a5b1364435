"""Cases for the matrix operators of a token model: the gated feed-forward block with its gradient, and the
orthogonalisation of an update by Newton-Schulz products.

Both work node by node, as the rest of the package does: the matrices of node i are a slice of row i of a float32 matrix
(or a 16-bit copy of it), its activations are ``rows`` vectors of ``d`` values.

Definitions (per node; Wg, Wu of f x d, Wd of d x f; act is silu(v) = v / (1 + e^-v), gelu(v) = v (1 + erf(v / sqrt 2)) / 2
or relu):

  block       g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T
  its grad    dh = dy Wd, du = dh act(g), dg = dh u act'(g); dWd = dy^T h, dWg = dg^T x, dWu = du^T x,
              dx = dg Wg + du Wu; g and u as the forward pass kept them
  orth        X = M / (|M| + eps) with the Frobenius norm, then five times X <- a X + (b A + c A A) X with A = X X^T
              ((a, b, c) = (3.4445, -4.7750, 2.0315): singular values go to about one); the result is s X
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
LARGEST = {"ff": 560e9, "ff_grad": 1130e9, "orth": 1370e9}   # flops of the largest listed cases; full precision takes several times as long


def listed():
    return [
        # one new token of a trained model: every weight read once, latency
        {"name": "block one token", "op": "ff", "nodes": 1, "rows": 1, "d": 1024, "f": 2816, "act": "silu", "type": "bf16", "weights": "bf16", "keep": False},
        # some sequences that a trained model answers together; weights straight from the float32 state
        {"name": "block few tokens", "op": "ff", "nodes": 1, "rows": 24, "d": 2048, "f": 5632, "act": "silu", "type": "bf16", "weights": "f32", "keep": False},
        # the toy model in full precision, no size even
        {"name": "block small odd", "op": "ff", "nodes": 2, "rows": 77, "d": 129, "f": 333, "act": "gelu", "type": "f32", "weights": "f32", "keep": True},
        # a training step of eight nodes, 4096 tokens each
        {"name": "block 8 nodes", "op": "ff", "nodes": 8, "rows": 4096, "d": 1024, "f": 2816, "act": "silu", "type": "bf16", "weights": "bf16", "keep": True},
        # full precision at the size of a small language model
        {"name": "block f32", "op": "ff", "nodes": 1, "rows": 4096, "d": 768, "f": 2048, "act": "gelu", "type": "f32", "weights": "f32", "keep": True},
        # gradient of a training step of eight nodes
        {"name": "block grad 8 nodes", "op": "ff_grad", "nodes": 8, "rows": 4096, "d": 1024, "f": 2816, "act": "silu", "type": "bf16", "weights": "bf16"},
        # gradient of short batches whose sizes fit no tile and no vector access
        {"name": "block grad odd", "op": "ff_grad", "nodes": 2, "rows": 501, "d": 515, "f": 1373, "act": "gelu", "type": "f16", "weights": "f16"},
        # gradient in full precision
        {"name": "block grad f32", "op": "ff_grad", "nodes": 1, "rows": 2048, "d": 768, "f": 2048, "act": "silu", "type": "f32", "weights": "f32"},
        # updates of the toy model's matrices on four nodes: latency
        {"name": "orth small", "op": "orth", "nodes": 4, "r": 64, "c": 128, "type": "f32"},
        # momenta of one feed-forward matrix on eight nodes, in the state's precision
        {"name": "orth 8 nodes", "op": "orth", "nodes": 8, "r": 1024, "c": 2816, "type": "f32"},
        # tall, odd, 16 bits
        {"name": "orth tall odd", "op": "orth", "nodes": 2, "r": 1373, "c": 515, "type": "f16"},
        # the widest square matrix of a large model, kept in 16 bits
        {"name": "orth large", "op": "orth", "nodes": 1, "r": 4096, "c": 4096, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: any operator, sizes spread over the logarithm, odd as often as round."""
    op = rng.choice(["ff", "ff_grad", "orth"])
    nodes = rng.choice([1, 1, 2, 4, 8])
    dt = rng.choice(["f32", "bf16", "f16"])
    even = rng.random() < 0.6

    def size(lo, hi):
        n = _log_int(rng, lo, hi)
        return max(64, n // 64 * 64) if even else n

    if op == "orth":
        r = size(48, 4096)
        c = min(4096, max(48, size(max(48, r // 6), min(4096, 6 * r))))
        case = {"op": op, "nodes": nodes, "r": r, "c": c, "type": dt}
        while work(case)["flops"] > LARGEST[op] / (3 if dt == "f32" else 1) or case["nodes"] * r * c > 3e7:
            case["nodes"] //= 2
        return case
    d = size(64, 2048)
    f = size(int(1.3 * d), 4 * d)
    nodes = max(1, min(nodes, int(2.5e7 // (d * f))))
    case = {"op": op, "nodes": nodes, "rows": 1, "d": d, "f": f, "act": rng.choice(["silu", "silu", "gelu", "relu"]), "type": dt, "weights": dt}
    if op == "ff":
        case["keep"] = rng.random() < 0.6
        if rng.random() < 0.3:
            case["weights"] = "f32"
    most = min(16384, 6e7 // (nodes * f), LARGEST[op] / (6 if dt == "f32" else 1) // work(case)["flops"])
    case["rows"] = _log_int(rng, 1, max(1, int(most)))
    return case


def work(case):
    n, e = case["nodes"], SIZE[case["type"]]
    if case["op"] == "orth":
        m, k = min(case["r"], case["c"]), max(case["r"], case["c"])
        # A and A A are symmetric: half of each is enough
        return {"bytes": 2 * n * m * k * e, "flops": n * STEPS * (m * (m + 1) * k + m * (m + 1) * m + 2 * m * m * k)}
    t, d, f, w = case["rows"], case["d"], case["f"], SIZE[case["weights"]]
    if case["op"] == "ff":
        return {"bytes": n * (3 * d * f * w + 2 * t * d * e + (2 * t * f * e if case["keep"] else 0)), "flops": 6 * n * t * d * f}
    return {"bytes": n * (6 * d * f * w + 3 * t * d * e + 2 * t * f * e), "flops": 12 * n * t * d * f}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)

    n, dt = case["nodes"], TYPES[case["type"]]
    s = {"case": case}
    if case["op"] == "orth":
        # a momentum: some directions that all batches share, weaker ones behind them, and the noise of single batches
        r, c = case["r"], case["c"]
        k = max(1, min(r, c) // 4)
        strength = torch.arange(1, k + 1, device="cuda").float().rsqrt()
        m = torch.bmm(normal(n, r, k) * strength, normal(n, k, c)) + normal(n, r, c, std=0.5)
        s["update"] = (m * 1e-4).to(dt)
        s["scale"] = math.sqrt(max(1.0, r / c))
        s["out"] = torch.empty((n, r, c), dtype=dt, device="cuda")
        return s
    t, d, f, wt = case["rows"], case["d"], case["f"], TYPES[case["weights"]]
    # after a norm: rows of about unit variance, some columns stronger than others
    s["x"] = (normal(n, t, d) * (0.5 + torch.rand((n, 1, d), generator=gen, device="cuda"))).to(dt)
    s["gate"] = normal(n, f, d, std=d ** -0.5).to(wt)
    s["up"] = normal(n, f, d, std=d ** -0.5).to(wt)
    s["down"] = normal(n, d, f, std=f ** -0.5).to(wt)
    if case["op"] == "ff_grad":
        s["g"] = torch.bmm(s["x"].float(), s["gate"].float().mT).to(dt)
        s["u"] = torch.bmm(s["x"].float(), s["up"].float().mT).to(dt)
        # 16-bit floats as a loss scale leaves them
        s["dy"] = normal(n, t, d, std=0.05 if dt is torch.float16 else 1e-3).to(dt)
    return s


def _act(v, kind):
    if kind == "silu":
        return v / (1.0 + torch.exp(-v))
    if kind == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return torch.where(v > 0, v, torch.zeros_like(v))


def _act_slope(v, kind):
    if kind == "silu":
        sig = 1.0 / (1.0 + torch.exp(-v))
        return sig * (1.0 + v * (1.0 - sig))
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))
    return (v > 0).to(v.dtype)


def _plain_block(s):
    dt, kind = TYPES[s["case"]["type"]], s["case"]["act"]
    x = s["x"].float()
    g, u = torch.bmm(x, s["gate"].float().mT), torch.bmm(x, s["up"].float().mT)
    y = torch.bmm(_act(g, kind) * u, s["down"].float().mT)
    return {"y": y.to(dt), "g": g.to(dt), "u": u.to(dt)} if s["case"]["keep"] else {"y": y.to(dt)}


def _plain_block_grad(s):
    dt, wt, kind = TYPES[s["case"]["type"]], TYPES[s["case"]["weights"]], s["case"]["act"]
    x, g, u, dy = (s[k].float() for k in ("x", "g", "u", "dy"))
    gate, up, down = (s[k].float() for k in ("gate", "up", "down"))
    a = _act(g, kind)
    dh = torch.bmm(dy, down)
    du, dg = dh * a, dh * u * _act_slope(g, kind)
    return {"dx": (torch.bmm(dg, gate) + torch.bmm(du, up)).to(dt), "dgate": torch.bmm(dg.mT, x).to(wt),
            "dup": torch.bmm(du.mT, x).to(wt), "ddown": torch.bmm(dy.mT, a * u).to(wt)}


def _plain_orth(s):
    m = s["update"].float()
    tall = m.shape[1] > m.shape[2]
    x = m.mT if tall else m
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = torch.bmm(x, x.mT)
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return (s["scale"] * (x.mT if tall else x)).to(s["update"].dtype)


def run(s):
    case = s["case"]
    if own:
        import paper_2105_09080_b200 as gpga
        if case["op"] == "ff":
            y, g, u = gpga.feed_forward_forward(s["x"], s["gate"], s["up"], s["down"], activation=case["act"], keep=case["keep"])
            return {"y": y, "g": g, "u": u} if case["keep"] else {"y": y}
        if case["op"] == "ff_grad":
            dx, dgate, dup, ddown = gpga.feed_forward_backward(s["dy"], s["x"], s["g"], s["u"], s["gate"], s["up"], s["down"],
                                                               activation=case["act"])
            return {"dx": dx, "dgate": dgate, "dup": dup, "ddown": ddown}
        return gpga.orthogonalize(s["update"], steps=STEPS, coefficients=COEFFICIENTS, scale=s["scale"], eps=EPS, out=s["out"])
    if case["op"] == "ff":
        return _plain_block(s)
    return _plain_block_grad(s) if case["op"] == "ff_grad" else _plain_orth(s)


def exact(case, seed):
    """The definitions in 64 bits, node by node."""
    s = prepare(case, seed)
    if case["op"] == "orth":
        a, b, c = COEFFICIENTS
        out = []
        for m in s["update"].double():
            z = m / (torch.linalg.matrix_norm(m) + EPS)
            eye = torch.eye(min(m.shape), dtype=torch.float64, device=m.device)
            for _ in range(STEPS):   # the polynomial of the gram matrix on the smaller side
                q = z @ z.T if m.shape[0] <= m.shape[1] else z.T @ z
                p = a * eye + q @ (b * eye + c * q)
                z = p @ z if m.shape[0] <= m.shape[1] else z @ p
            out.append(s["scale"] * z)
        return torch.stack(out)
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[case["act"]]
    found = []
    for i in range(case["nodes"]):
        x, gate, up, down = (s[k][i].double() for k in ("x", "gate", "up", "down"))
        if case["op"] == "ff":
            g, u = x @ gate.T, x @ up.T
            y = (act(g) * u) @ down.T
            found.append({"y": y, "g": g, "u": u} if case["keep"] else {"y": y})
            continue
        g = s["g"][i].double().requires_grad_()
        u, dy = s["u"][i].double(), s["dy"][i].double()
        with torch.enable_grad():
            v = act(g)
            slope, = torch.autograd.grad(v.sum(), g)
        v = v.detach()
        dh = dy @ down
        found.append({"dx": (dh * u * slope) @ gate + (dh * v) @ up, "dgate": (x.T @ (dh * u * slope)).T,
                      "dup": (x.T @ (dh * v)).T, "ddown": ((v * u).T @ dy).T})
    return {k: torch.stack([r[k] for r in found]) for k in found[0]}
