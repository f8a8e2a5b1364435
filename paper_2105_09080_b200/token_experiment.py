"""A token model trained by Gossip-PGA: embedding lookups, dropout, layer norm and their gradients node by node.

    python -m paper_2105_09080_b200.token_experiment [--nodes 8] [--iters 400] [--every 50] [--dtype bf16]

Every node i holds all parameters of a next-token model in row i of X,

    z = B_i[tok_{t-1}] + dropout(A_i[tok_t]),   y = layer_norm(z; w_i, b_i),   logits = y C_i^T,

(A, B, C tables of vocab x dim) and draws its own mini-batches: a node sees some words more often than the others do,
the rule that makes the next word from the last two is common.  One iteration is Algorithm 1's: the gradient of the
mean cross-entropy at every node, written into the same places of G, the local update x_i - gamma g_i, and a gossip
step on the ring or the one-peer exponential graph, or every H-th time the global average.  The lookups, the dropout,
the norm, their gradients and the mixing are the library's; the two matrix products per direction and the softmax
between them are torch's.  Prints one JSON line per method: mean loss over the nodes, loss of the node average without
dropout, and consensus distance versus iteration.
"""
from __future__ import annotations

import argparse
import json
import math

from . import binding as B


class TokenModel:
    """n nodes' parameters in rows of X, their gradients in rows of G (same places), and the mixing handle."""

    def __init__(self, n, vocab, dim, topology, H, seed, device="cuda", dtype=None):
        import torch
        if dim % 8:
            raise ValueError("dim must be a multiple of 8")
        self.n, self.vocab, self.dim, self.seed = n, vocab, dim, seed
        self.dtype = dtype or torch.float32
        table = vocab * dim
        self.d = 3 * table + 2 * dim
        ld = (self.d + 31) // 32 * 32                      # rows start on 128-byte lines
        self.X = torch.zeros((n, ld), device=device)
        self.G = torch.zeros((n, ld), device=device)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        row = torch.randn(self.d, generator=gen, device=device) / math.sqrt(dim)
        row[3 * table:3 * table + dim] = 1.0
        row[3 * table + dim:] = 0.0
        self.X[:, :self.d] = row                           # Algorithm 1: equal initial rows
        # The mixing alone: learning rate 0 leaves the half-step of the library's quadratic objective at X, whose local
        # update is done before the call; in place (one buffer for X and X+), G stands in for the data, which is read and
        # multiplied by zero: an infinite gradient leaves NaN in the rows it reaches.
        self.mixer = B.Gpga(n, self.d, topology, H, 0.0, seed)
        self.mixer.set_row_stride(ld)
        self.mixer.bind(self.X, self.X, self.G)

    def slices(self, M):
        """(A, B, C, weight, bias) inside the rows of X or G."""
        t, d = self.vocab * self.dim, self.dim
        tables = [M[:, i * t:(i + 1) * t].unflatten(1, (self.vocab, d)) for i in range(3)]
        return (*tables, M[:, 3 * t:3 * t + d], M[:, 3 * t + d:3 * t + 2 * d])

    def gradient(self, k, before, cur, target, p):
        """Fills G with every node's gradient on its batch (nodes, T of tokens each); returns the nodes' losses."""
        import torch
        from .token_ops import embedding_backward, embedding_forward, layer_norm_backward, layer_norm_forward
        A, Bt, Ct, w, b = self.slices(self.X)
        dA, dB, dC, dw, db = self.slices(self.G)
        n, T = cur.shape
        mask = {"p": p, "seed": self.seed, "k": k, "site": 0, "nodes": n}
        x = embedding_forward(A, cur, dtype=self.dtype)
        r = embedding_forward(Bt, before, dtype=self.dtype)
        y, z, mean, rstd = layer_norm_forward(x, w, b, residual=r, out=x, z=r, **mask)
        logits = torch.bmm(y.float(), Ct.transpose(1, 2))
        logp = torch.log_softmax(logits, -1)
        loss = -logp.gather(2, target.unsqueeze(2)).mean((1, 2))
        dlogits = logp.exp_()
        dlogits.scatter_add_(2, target.unsqueeze(2), torch.full_like(target, -1, dtype=torch.float32).unsqueeze(2))
        dlogits /= T
        dC.copy_(torch.bmm(dlogits.transpose(1, 2), y.float()))
        dy = torch.bmm(dlogits, Ct).to(self.dtype)
        dr, dx, _, _ = layer_norm_backward(dy, z, mean, rstd, w, dresidual=dy, dweight=dw, dbias=db, **mask)
        embedding_backward(dx, cur, dA)
        embedding_backward(dr, before, dB)
        return loss

    def step(self, k, gamma):
        """Local update with the gradient in G, then the mix of iteration k."""
        self.X[:, :self.d].sub_(self.G[:, :self.d], alpha=gamma)
        self.mixer.step(k)

    def average_loss(self, before, cur, target):
        """Cross-entropy of the node average on all given batches, without dropout."""
        import torch
        from .token_ops import embedding_forward, layer_norm_forward
        A, Bt, Ct, w, b = (t[0] for t in self.slices(self.X.mean(0, keepdim=True)))
        x = embedding_forward(A, cur, dtype=self.dtype)
        y = layer_norm_forward(x, w, b, residual=embedding_forward(Bt, before, dtype=self.dtype))[0]
        return torch.nn.functional.cross_entropy((y.float() @ Ct.t()).flatten(0, 1), target.flatten()).item()

    def close(self):
        self.mixer.close()


def batch(n, T, vocab, k, seed, device="cuda"):
    """(before, cur, target), each (n, T): node i draws three words in four from its own part of the vocabulary, the
    next word is a fixed function of the last two, replaced by any word one time in ten."""
    import torch
    gen = torch.Generator(device=device)
    gen.manual_seed(seed * 1000003 + k)
    part = max(1, vocab // n)
    own = torch.arange(n, device=device).view(n, 1, 1) * part
    words = torch.randint(0, vocab, (n, T, 2), generator=gen, device=device)
    local = torch.rand((n, T, 2), generator=gen, device=device) < 0.75
    words = torch.where(local, (own + words % part) % vocab, words)
    before, cur = words[..., 0].contiguous(), words[..., 1].contiguous()
    target = (cur * 3 + (before % 4) * 5 + 1) % vocab
    noise = torch.rand((n, T), generator=gen, device=device) < 0.1
    return before, cur, torch.where(noise, torch.randint(0, vocab, (n, T), generator=gen, device=device), target)


def train(name, topology, H, n=8, T=512, vocab=256, dim=128, iters=400, every=50, gamma=1.0, p=0.1, seed=20210509, dtype=None):
    m = TokenModel(n, vocab, dim, topology, H, seed, dtype=dtype)
    test = batch(n, 2 * T, vocab, 0, seed + 1)
    traj = []
    for k in range(iters):
        loss = m.gradient(k, *batch(n, T, vocab, k, seed), p)
        m.step(k, gamma)
        if (k + 1) % every == 0 or k + 1 == iters:
            traj.append({"k": k + 1, "loss": loss.mean().item(), "average_loss": m.average_loss(*test),
                         "consensus": m.mixer.consensus_distance()})
    m.close()
    return {"method": name, "H": H or "inf", "nodes": n, "tokens_per_node": T, "vocab": vocab, "dim": dim, "gamma": gamma,
            "dropout": p, "trajectory": traj}


METHODS = (("parallel SGD", B.GPGA_TOPO_RING, 1), ("Gossip SGD, ring", B.GPGA_TOPO_RING, 0), ("Gossip-PGA, ring", B.GPGA_TOPO_RING, 16),
           ("Gossip-PGA, one-peer exp", B.GPGA_TOPO_EXP, 16), ("Local SGD", B.GPGA_TOPO_NONE, 16))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--nodes", type=int, default=8)
    ap.add_argument("--iters", type=int, default=400)
    ap.add_argument("--every", type=int, default=50)
    ap.add_argument("--tokens", type=int, default=512, help="per node and iteration")
    ap.add_argument("--vocab", type=int, default=256)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--gamma", type=float, default=1.0)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--dtype", choices=("f32", "bf16", "f16"), default="f32")
    args = ap.parse_args(argv)
    import torch
    if not torch.cuda.is_available():
        raise RuntimeError("the experiment needs a CUDA device (there is no CPU fallback)")
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[args.dtype]
    for name, topology, H in METHODS:
        print(json.dumps(train(name, topology, H, args.nodes, args.tokens, args.vocab, args.dim, args.iters, args.every, args.gamma,
                               args.dropout, dtype=dtype)), flush=True)


if __name__ == "__main__":
    main()
