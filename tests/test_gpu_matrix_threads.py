"""Matrix operators in a fresh process: the library's first calls inside a graph capture, and from several host threads at
once, each on a stream of its own."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

HEAD = """
import threading
import torch
import paper_2105_09080_b200 as pkg

torch.cuda.init()
pkg.lib()


def inputs(seed, n, t, d, f, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    make = lambda *s: torch.empty(s, device="cuda").normal_(0.0, 0.3, generator=g).to(dtype)
    return make(n, t, d), make(n, f, d), make(n, f, d), make(n, d, f)


def work(x, gate, up, down):
    y, g, u = pkg.feed_forward_forward(x, gate, up, down)
    few = pkg.feed_forward_forward(x[:, :5].contiguous(), gate, up, down, keep=False)[0]
    return [y, g, u, few, *pkg.feed_forward_backward(y, x, g, u, gate, up, down), pkg.orthogonalize(gate), pkg.orthogonalize(gate[:, :40])]


SHAPES = [(1, 2, 100, 64, 96, torch.float32), (2, 2, 300, 200, 264, torch.bfloat16), (3, 1, 700, 129, 333, torch.float16), (4, 1, 64, 150, 180, torch.float32)]
"""

CAPTURE = HEAD + """
made = [inputs(*s) for s in SHAPES]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = [work(*m) for m in made]
graph.replay()
torch.cuda.synchronize()
for m, r in zip(made, got):
    assert all(torch.equal(a, b) for a, b in zip(work(*m), r))
pkg.token_status()
print("same")
"""

THREADS = HEAD + """
made = [inputs(*s) for s in SHAPES]
torch.cuda.synchronize()
start = threading.Barrier(4)
results, errors = [None] * 4, []


def run(i):
    try:
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            out = []
            for m in made:
                start.wait(60)
                out.append(work(*m))
            stream.synchronize()
        results[i] = out
    except BaseException as e:
        errors.append(repr(e))
        start.abort()


threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
[t.start() for t in threads]
[t.join() for t in threads]
assert not errors, errors
for j, m in enumerate(made):
    want = work(*m)
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(want, r[j]))
pkg.token_status()
print("same")
"""


@pytest.mark.parametrize("script", [CAPTURE, THREADS], ids=["capture", "threads"])
def test_first_calls(script):
    root = Path(__file__).resolve().parent.parent
    out = subprocess.run([sys.executable, "-c", script], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.split() == ["same"], out.stderr[-2000:]
