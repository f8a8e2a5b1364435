"""Cases for the token-block operators: embedding lookup and its gradient, dropout from a counter-based
generator, layer norm (with the residual sum and the dropout in front of it) and its gradient.

Every operator works node by node, as the rest of the package does: the parameters of node i are a slice of
row i of a float32 matrix, and its activations are ``rows`` vectors of ``d`` values.

Definitions (W_i, w_i, b_i: parameters of node i; all sums over one row unless stated):

  lookup      out[i,t,:] = s W_i[tok[i,t],:]; a token outside [0, vocab) gives a zero row
  its grad    dW_i[v,:] = s sum over t with tok[i,t] = v of dout[i,t,:]
  dropout     column j of row t of node i belongs to the Philox4x32-10 call with key (seed low, seed high) and
              counter (t ceil(d/8) + (j >> 3), i, k, 2^30 + site); its 16 bits are half j & 1 (low half first) of
              word (j & 7) >> 1.  With q = floor(65536 p + 1/2) it is kept where these bits are at least q and then
              multiplied by 65536 / (65536 - q), and exactly zero elsewhere
  norm        z = residual + dropout(x), mean and rstd = 1 / sqrt(variance + eps) of z, y = (z - mean) rstd w_i + b_i
  its grad    xh = (z - mean) rstd, h = w_i dy, g = rstd (h - mean(h) - xh mean(h xh)) + dz;
              dresidual = g, dx = dropout(g) with the same mask, dw_i = sum over rows of dy xh, db_i = sum of dy
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
SITE0 = 1 << 30


def listed():
    return [
        # the lookup of one new token, as when a trained model answers: latency
        {"name": "lookup one token", "op": "lookup", "nodes": 1, "rows": 1, "d": 1024, "vocab": 32000, "type": "bf16"},
        # the lookup of a training step of eight nodes, 4096 tokens each
        {"name": "lookup 8 nodes", "op": "lookup", "nodes": 8, "rows": 4096, "d": 1024, "vocab": 32000, "type": "bf16"},
        # gradient of a toy model: odd width, few tokens, full precision
        {"name": "lookup grad small odd", "op": "lookup_grad", "nodes": 1, "rows": 37, "d": 257, "vocab": 1021, "type": "f32"},
        # gradient of short batches on eight nodes: nearly all of it is rows that no token touched
        {"name": "lookup grad 8 nodes", "op": "lookup_grad", "nodes": 8, "rows": 512, "d": 1024, "vocab": 32000, "type": "bf16"},
        # gradient of one node's large batch, word frequencies falling as 1 / rank
        {"name": "lookup grad large", "op": "lookup_grad", "nodes": 1, "rows": 65536, "d": 1024, "vocab": 50021, "type": "bf16"},
        # dropout of a short sequence of a narrow model
        {"name": "dropout small odd", "op": "dropout", "nodes": 1, "rows": 19, "d": 333, "type": "f32", "p": 0.1},
        # dropout of the widest activations of a step: four times the model's width
        {"name": "dropout large", "op": "dropout", "nodes": 8, "rows": 4096, "d": 4096, "type": "bf16", "p": 0.1},
        # layer norm of one new token: latency
        {"name": "norm one token", "op": "norm", "nodes": 1, "rows": 1, "d": 1024, "type": "bf16", "p": 0.0, "residual": True},
        # the edge of a residual block in a training step of eight nodes
        {"name": "norm 8 nodes", "op": "norm", "nodes": 8, "rows": 4096, "d": 1024, "type": "bf16", "p": 0.1, "residual": True},
        # a width that no vector access divides
        {"name": "norm odd", "op": "norm", "nodes": 2, "rows": 5001, "d": 1023, "type": "f16", "p": 0.0, "residual": False},
        # gradient of the residual block's edge in a training step of eight nodes
        {"name": "norm grad 8 nodes", "op": "norm_grad", "nodes": 8, "rows": 4096, "d": 1024, "type": "bf16", "p": 0.1, "residual": True},
        # gradient of a wide model's layer norm in full precision
        {"name": "norm grad wide", "op": "norm_grad", "nodes": 1, "rows": 2000, "d": 8192, "type": "f32", "p": 0.0, "residual": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: any operator, sizes spread over the logarithm, widths that are odd as often as round."""
    op = rng.choice(["lookup", "lookup_grad", "dropout", "norm", "norm_grad"])
    nodes = rng.choice([1, 1, 2, 4, 8, 12])
    d = _log_int(rng, 48, 8192)
    if rng.random() < 0.6:
        d = max(64, d // 64 * 64)
    rows = _log_int(rng, 1, max(1, min(65536, 32_000_000 // (nodes * d))))
    case = {"op": op, "nodes": nodes, "rows": rows, "d": d, "type": rng.choice(["f32", "bf16", "f16"])}
    if op in ("lookup", "lookup_grad"):
        case["vocab"] = _log_int(rng, 100, min(100_000, 200_000_000 // (nodes * d)))
    else:
        case["p"] = rng.choice([0.1, round(rng.uniform(0.01, 0.6), 3)]) if op == "dropout" or rng.random() < 0.6 else 0.0
    if op in ("norm", "norm_grad"):
        case["residual"] = rng.random() < 0.6
    return case


def _frequencies(vocab):
    """Word frequencies of natural text: 1 / rank, normalised."""
    f = 1.0 / torch.arange(1, vocab + 1, dtype=torch.float64)
    return f / f.sum()


def work(case):
    n, t, d, e = case["nodes"], case["rows"], case["d"], SIZE[case["type"]]
    N = n * t * d
    if case["op"] in ("lookup", "lookup_grad"):
        if case["op"] == "lookup":   # distinct table rows once, tokens, outputs
            f = _frequencies(case["vocab"])
            distinct = float((1.0 - torch.exp(t * torch.log1p(-f))).sum()) if case["vocab"] > 1 else 1.0
            return {"bytes": int(n * distinct * d * 4 + n * t * 8 + N * e), "flops": N}
        return {"bytes": N * e + n * t * 8 + n * case["vocab"] * d * 4, "flops": N}
    if case["op"] == "dropout":
        return {"bytes": 2 * N * e, "flops": N}
    rest = 2 * n * t * 4 + 2 * n * d * 4
    if case["op"] == "norm":
        mixed = case["residual"] or case["p"] > 0
        return {"bytes": N * e * (2 + case["residual"] + mixed) + rest, "flops": 9 * N}
    # dy, z, (dz) read, g and, with dropout, dx written; mean, rstd and w read, dw and db written
    return {"bytes": N * e * (3 + case["residual"] + (case["p"] > 0)) + rest + n * d * 4, "flops": 14 * N}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, t, d, dt = case["nodes"], case["rows"], case["d"], TYPES[case["type"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)

    s = {"case": case, "seed": 1000003 * seed + 17, "k": seed % 1000, "site": 3}
    if case["op"] in ("lookup", "lookup_grad"):
        V = case["vocab"]
        # the words of a vocabulary are in no order of frequency
        rank = torch.randperm(V, generator=g, device="cuda")
        u = torch.rand((n, t), generator=g, device="cuda", dtype=torch.float64)
        s["tokens"] = rank[torch.searchsorted(_frequencies(V).cumsum(0).cuda(), u).clamp_(max=V - 1)]
        s["scale"] = math.sqrt(d)
        if case["op"] == "lookup":
            s["table"] = normal(n, V, d, std=0.02)
            s["out"] = torch.empty((n, t, d), dtype=dt, device="cuda")
        else:
            s["dout"] = normal(n, t, d, std=1e-3, dtype=dt)
            s["grad"] = torch.empty((n, V, d), device="cuda")
        return s
    if case["op"] == "dropout":
        s["x"] = normal(n, t, d, dtype=dt)
        s["out"] = torch.empty_like(s["x"])
        return s
    s["weight"] = normal(n, d, std=0.1, mean=1.0)
    s["bias"] = normal(n, d, std=0.1)
    # rows differ in their level and spread
    x = normal(n, t, d) * (0.5 + torch.rand((n, t, 1), generator=g, device="cuda")) + normal(n, t, 1, std=0.5)
    if case["op"] == "norm":
        s["x"] = x.to(dt)
        s["residual"] = normal(n, t, d, std=1.5, dtype=dt) if case["residual"] else None
        s["out"] = torch.empty_like(s["x"])
        s["z"] = torch.empty_like(s["x"]) if case["residual"] or case["p"] > 0 else None
        s["mean"], s["rstd"] = torch.empty((2, n, t), device="cuda").unbind(0)
        return s
    s["z"] = x.to(dt)
    s["mean"] = x.mean(-1)
    s["rstd"] = torch.rsqrt(x.var(-1, unbiased=False) + EPS)
    s["dy"] = normal(n, t, d, std=1e-2, dtype=dt)
    s["dz"] = normal(n, t, d, std=1e-2, dtype=dt) if case["residual"] else None
    s["dresidual"] = torch.empty_like(s["z"])
    s["dx"] = torch.empty_like(s["z"]) if case["p"] > 0 else None
    s["dweight"], s["dbias"] = torch.empty((2, n, d), device="cuda").unbind(0)
    return s


# ---- the plain forms -----------------------------------------------------------------------------
def _mulhilo(a, m):
    """High and low 32-bit words of a * m for a < 2^32 held in int64 and a constant m < 2^32."""
    low = (a & 0xFFFF) * m
    high = (a >> 16) * m + (low >> 16)
    return high >> 16, ((high & 0xFFFF) << 16) | (low & 0xFFFF)


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 on int64 tensors that hold 32-bit words."""
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        h0, l0 = _mulhilo(c0, 0xD2511F53)
        h1, l1 = _mulhilo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def _dropped(x, s):
    """dropout(x) in float32 for x (nodes, rows, d)."""
    n, t, d = x.shape
    q = int(math.floor(65536 * s["case"]["p"] + 0.5))
    groups = -(-d // 8)
    c0 = torch.arange(t * groups, device=x.device).view(1, t, groups).expand(n, t, groups)
    c1 = torch.arange(n, device=x.device).view(n, 1, 1).expand(n, t, groups)
    c2, c3 = torch.full_like(c0, s["k"]), torch.full_like(c0, SITE0 + s["site"])
    words = torch.stack(_philox(c0, c1, c2, c3, s["seed"]), -1)
    bits = torch.stack((words & 0xFFFF, words >> 16), -1).reshape(n, t, groups * 8)[..., :d]
    return torch.where(bits >= q, x.float() * (65536.0 / (65536 - q)), torch.zeros((), device=x.device))


def _plain(s):
    case = s["case"]
    n, t, d, dt = case["nodes"], case["rows"], case["d"], TYPES[case["type"]]
    if case["op"] == "lookup":
        node = torch.arange(n, device="cuda").view(n, 1)
        return [(s["table"][node, s["tokens"]] * s["scale"]).to(dt)]
    if case["op"] == "lookup_grad":
        V = case["vocab"]
        grad = torch.zeros((n * V, d), device="cuda")
        at = s["tokens"] + V * torch.arange(n, device="cuda").view(n, 1)
        grad.index_add_(0, at.view(-1), s["dout"].float().view(n * t, d) * s["scale"])
        return [grad.view(n, V, d)]
    if case["op"] == "dropout":
        return [_dropped(s["x"], s).to(dt)]
    w = s["weight"].view(n, 1, d)
    if case["op"] == "norm":
        z = _dropped(s["x"], s) if case["p"] > 0 else s["x"].float()
        if s["residual"] is not None:
            z = z + s["residual"].float()
        mean = z.mean(-1, keepdim=True)
        rstd = torch.rsqrt((z - mean).square().mean(-1, keepdim=True) + EPS)
        y = ((z - mean) * rstd * w + s["bias"].view(n, 1, d)).to(dt)
        stats = [mean.view(n, t), rstd.view(n, t)]
        return [y] + ([z.to(dt)] if s["z"] is not None else []) + stats
    dy = s["dy"].float()
    rstd = s["rstd"].unsqueeze(-1)
    xh = (s["z"].float() - s["mean"].unsqueeze(-1)) * rstd
    h = dy * w
    g = rstd * (h - h.mean(-1, keepdim=True) - xh * (h * xh).mean(-1, keepdim=True))
    if s["dz"] is not None:
        g = g + s["dz"].float()
    dx = [_dropped(g, s).to(dt)] if case["p"] > 0 else []
    return [g.to(dt)] + dx + [(dy * xh).sum(1), dy.sum(1)]


# ---- the package's calls -------------------------------------------------------------------------
def _own(s):
    import paper_2105_09080_b200 as pkg
    case = s["case"]
    if case["op"] == "lookup":
        return [pkg.embedding_forward(s["table"], s["tokens"], scale=s["scale"], out=s["out"])]
    if case["op"] == "lookup_grad":
        return [pkg.embedding_backward(s["dout"], s["tokens"], s["grad"], scale=s["scale"])]
    mask = {"p": case["p"], "seed": s["seed"], "k": s["k"], "site": s["site"], "nodes": case["nodes"]}
    if case["op"] == "dropout":
        return [pkg.dropout(s["x"], out=s["out"], **mask)]
    if case["op"] == "norm":
        y, z, mean, rstd = pkg.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=EPS, residual=s["residual"], out=s["out"],
                                                  z=s["z"], mean=s["mean"], rstd=s["rstd"], **mask)
        return [y] + ([z] if s["z"] is not None else []) + [mean, rstd]
    g, dx, dw, db = pkg.layer_norm_backward(s["dy"], s["z"], s["mean"], s["rstd"], s["weight"], dz=s["dz"], dresidual=s["dresidual"],
                                            dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"], **mask)
    return [g] + ([dx] if s["dx"] is not None else []) + [dw, db]


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _kept(case, s):
    """The factor of every element, in float64: 0 or 65536 / (65536 - q).  One node at a time, the generator written
    out for unsigned words of numpy."""
    import numpy as np
    n, t, d = case["nodes"], case["rows"], case["d"]
    q = math.floor(65536 * case["p"] + 0.5)
    groups = (d + 7) // 8
    low = np.uint64(0xFFFFFFFF)
    w32 = np.uint64(32)
    out = []
    for i in range(n):
        ctr = [np.arange(t * groups, dtype=np.uint64), np.uint64(i), np.uint64(s["k"]), np.uint64(SITE0 + s["site"])]
        key = [s["seed"] % 2**32, s["seed"] // 2**32 % 2**32]
        for r in range(10):
            a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
            ctr = [(b >> w32) ^ ctr[1] ^ np.uint64(key[0]), b & low, (a >> w32) ^ ctr[3] ^ np.uint64(key[1]), a & low]
            key = [(key[0] + 0x9E3779B9) % 2**32, (key[1] + 0xBB67AE85) % 2**32]
        bits = np.empty((t * groups, 8), dtype=np.uint16)
        for c in range(4):
            word = np.broadcast_to(ctr[c], (t * groups,))
            bits[:, 2 * c] = word & np.uint64(0xFFFF)
            bits[:, 2 * c + 1] = word >> np.uint64(16)
        out.append(torch.from_numpy(bits.reshape(t, groups * 8)[:, :d] >= q))
    return torch.stack(out).cuda().double() * (65536.0 / (65536 - q))


def exact(case, seed):
    s = prepare(case, seed)
    n, t, d = case["nodes"], case["rows"], case["d"]
    if case["op"] == "lookup":
        return [torch.stack([s["table"][i].index_select(0, s["tokens"][i]).double() for i in range(n)]) * s["scale"]]
    if case["op"] == "lookup_grad":
        if n * case["vocab"] * d > 300_000_000:
            return None
        grads = []
        for i in range(n):   # rows in the order of their tokens, then differences of running sums of 64 bits
            order = torch.argsort(s["tokens"][i], stable=True)
            words, counts = torch.unique_consecutive(s["tokens"][i][order], return_counts=True)
            ends = counts.cumsum(0)
            dense = torch.zeros((case["vocab"], d), dtype=torch.float64, device="cuda")
            for c in range(0, d, 256):
                total = s["dout"][i][order, c:c + 256].double().cumsum(0)[ends - 1]
                dense[words, c:c + 256] = torch.cat([total[:1], total[1:] - total[:-1]])
            grads.append(dense * s["scale"])
        return [torch.stack(grads)]
    if case["op"] == "dropout":
        return [s["x"].double() * _kept(case, s)]
    w, b = s["weight"].double()[:, None], s["bias"].double()[:, None]
    keep = _kept(case, s) if case["p"] > 0 else 1.0
    if case["op"] == "norm":
        z = s["x"].double() * keep + (s["residual"].double() if case["residual"] else 0.0)
        var, mean = torch.var_mean(z, -1, correction=0, keepdim=True)
        y = torch.addcmul(b, (z - mean) / (var + EPS).sqrt(), w)
        return [y] + ([z] if s["z"] is not None else []) + [mean[..., 0], (var[..., 0] + EPS) ** -0.5]
    dy, r = s["dy"].double(), s["rstd"].double()[..., None]
    xh = (s["z"].double() - s["mean"].double()[..., None]) * r
    a = torch.einsum("ntd,nd->nt", dy, s["weight"].double())[..., None] / d
    c = torch.einsum("ntd,ntd,nd->nt", dy, xh, s["weight"].double())[..., None] / d
    g = r * (w * dy - a - c * xh) + (s["dz"].double() if case["residual"] else 0.0)
    return [g] + ([g * keep] if case["p"] > 0 else []) + [torch.einsum("ntd,ntd->nd", dy, xh), dy.sum(1)]
