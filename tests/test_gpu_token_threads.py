"""Token-block operators called from several host threads at once, from the library's first launches on."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

SCRIPT = """
import threading
import torch
import paper_2105_09080_b200 as pkg

THREADS = 4
torch.cuda.init()
pkg.lib()


def inputs(d, rows):
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    x = torch.empty((2, rows, d), device="cuda").normal_(generator=g)
    tokens = torch.randint(0, 300, (2, rows), generator=g, device="cuda")
    return x, torch.empty((2, d), device="cuda").normal_(generator=g), tokens


def work(x, w, tokens, stream):
    # rows off the alignment alike, unalike, and aligned without a bias: kernels whose grid goes by what an SM holds
    d = x.shape[-1]
    wide = torch.empty((2, x.shape[1], d + 3), dtype=x.dtype, device="cuda")[..., 1:1 + d]
    y, z, mean, rstd = pkg.layer_norm_forward(x, w, w, p=0.2, seed=5)
    other = pkg.layer_norm_forward(x, w, None, out=wide)[0]
    g, dx, dw, db = pkg.layer_norm_backward(y, z, mean, rstd, w, p=0.2, seed=5)
    grad = pkg.embedding_backward(dx, tokens, torch.empty((2, 300, d), device="cuda"))
    stream.synchronize()
    return [y, z, mean, rstd, other, g, dx, dw, db, grad]


shapes = [(d, 700) for d in (33, 71, 203, 333, 701, 1000, 1003, 1021, 1501, 1999, 2501, 3999, 5001, 64, 512, 8000)]
made = {s: inputs(*s) for s in shapes}
torch.cuda.synchronize()
start = threading.Barrier(THREADS)
results, errors = [None] * THREADS, []


def run(i):
    try:
        stream = torch.cuda.Stream()
        out = {}
        with torch.cuda.stream(stream):
            for s in shapes:
                start.wait(60)      # every shape's first calls at once
                out[s] = work(*made[s], stream)
        results[i] = out
    except BaseException as e:
        errors.append(repr(e))
        start.abort()


threads = [threading.Thread(target=run, args=(i,)) for i in range(THREADS)]
[t.start() for t in threads]
[t.join() for t in threads]
assert not errors, errors
torch.cuda.synchronize()
for s in shapes:
    want = work(*made[s], torch.cuda.current_stream())
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(want, r[s])), s
print("same")
"""


def test_first_calls_from_several_threads():
    """Every thread gets what one thread alone gets, bit for bit.  A process of its own, so that nothing is set up yet."""
    root = Path(__file__).resolve().parent.parent
    out = subprocess.run([sys.executable, "-c", SCRIPT], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.split() == ["same"], out.stderr[-2000:]
