"""Host-side checks of the matrix operators' C entries (gated feed-forward block, orthogonalisation): arguments are judged
before CUDA is touched, the binding packs the structs as a C compiler lays them out, and scratch is what the arguments need."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest
import torch

import paper_2105_09080_b200 as pkg
from paper_2105_09080_b200 import token_ops

ROOT = Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_2105_09080_b200" / "csrc"
A, B, C, D, S = 0x100000, 0x200000, 0x300000, 0x400000, 0x500000        # made-up aligned addresses, never read
F32, BF16, F16 = 0, 1, 2
MEMBERS = {
    "gpga_feed_forward_forward": "x gate up down y g u scratch scratch_bytes ldx ldgate node_gate ldup node_up lddown node_down ldy ldg ldu dtype "
                                 "weight_dtype activation nodes rows d f",
    "gpga_feed_forward_backward": "dy x g u gate up down dx dgate dup ddown scratch scratch_bytes lddy ldx ldg ldu ldgate node_gate ldup node_up lddown "
                                  "node_down lddx lddgate node_dgate lddup node_dup ldddown node_ddown dtype weight_dtype grad_dtype accumulate "
                                  "activation nodes rows d f",
    "gpga_orthogonalize": "update out scratch scratch_bytes ldm node_ldm ldo node_ldo dtype nodes r c steps accumulate c1 c3 c5 scale eps",
}
n, t, d, f = 2, 40, 16, 24
FORWARD = dict(x=A, gate=B, up=C, down=D, y=A, g=0, u=0, scratch=S, scratch_bytes=1 << 40, ldx=d, ldgate=d, node_gate=f * d, ldup=d, node_up=f * d,
               lddown=f, node_down=f * d, ldy=d, ldg=f, ldu=f, dtype=BF16, weight_dtype=BF16, activation=0, nodes=n, rows=t, d=d, f=f)
BACKWARD = dict(dy=A, x=A, g=A, u=A, gate=B, up=C, down=D, dx=A, dgate=B, dup=C, ddown=D, scratch=S, scratch_bytes=1 << 40, lddy=d, ldx=d, ldg=f, ldu=f,
                ldgate=d, node_gate=f * d, ldup=d, node_up=f * d, lddown=f, node_down=f * d, lddx=d, lddgate=d, node_dgate=f * d, lddup=d, node_dup=f * d,
                ldddown=f, node_ddown=f * d, dtype=BF16, weight_dtype=F32, grad_dtype=F32, accumulate=0, activation=1, nodes=n, rows=t, d=d, f=f)
ORTH = dict(update=A, out=B, scratch=S, scratch_bytes=1 << 40, ldm=600, node_ldm=500 * 600, ldo=600, node_ldo=500 * 600, dtype=F32, nodes=n, r=500, c=600,
            steps=5, accumulate=0, c1=3.4, c3=-4.8, c5=2.0, scale=1.0, eps=1e-7)
SAME_ROWS = {"gpga_feed_forward_forward": FORWARD, "gpga_feed_forward_backward": BACKWARD, "gpga_orthogonalize": ORTH}


@pytest.fixture(scope="module")
def L():
    return pkg.lib()


def packed(name, values):
    return token_ops.ARGS[name].pack(*(values[m] for m in MEMBERS[name].split()))


def refused(L, name, **changes):
    """Whether the entry refuses these arguments, with a text, and the scratch function has nothing to say but 0."""
    args = packed(name, {**SAME_ROWS[name], **changes})
    st = getattr(L, name)(args, None)
    return st == pkg.GPGA_ERR_INVALID_ARG and len(L.gpga_last_error(None)) > 0


def test_structs_are_packed_as_in_c(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    lines = []
    for name, members in MEMBERS.items():
        lines += [f'printf("%zu ", offsetof({name}_args_t, {m}));' for m in members.split()]
        lines.append(f'printf("%zu\\n", sizeof({name}_args_t));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gpga.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-I", str(ROOT / "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines()
    for (name, members), line in zip(MEMBERS.items(), out):
        count = len(members.split())
        assert [int(x) for x in line.split()] == [8 * i for i in range(count + 1)], name
        assert token_ops.ARGS[name].size == 8 * count
        assert getattr(pkg.lib(), name)(None, None) == pkg.GPGA_ERR_INVALID_ARG
        assert getattr(pkg.lib(), name + "_scratch_bytes")(None) == 0


@pytest.mark.parametrize("changes", [
    dict(x=0), dict(gate=0), dict(up=0), dict(down=0), dict(y=0), dict(g=A), dict(u=A), dict(scratch=0), dict(scratch=S + 8), dict(scratch_bytes=0),
    dict(ldx=d - 1), dict(ldgate=d - 1), dict(ldup=d - 1), dict(lddown=f - 1), dict(ldy=d - 1), dict(g=A, u=A, ldg=f - 1), dict(g=A, u=A, ldu=f - 1),
    dict(node_gate=-1), dict(ldx=2**41), dict(dtype=3), dict(dtype=-1), dict(dtype=2**32), dict(weight_dtype=F16), dict(weight_dtype=7),
    dict(dtype=F32), dict(activation=3), dict(activation=-1), dict(nodes=0), dict(nodes=65536), dict(rows=-1), dict(rows=2**30), dict(d=0),
    dict(d=2**20 + 1, ldx=2**21, ldgate=2**21, ldup=2**21, ldy=2**21), dict(f=0), dict(f=2**20 + 1, lddown=2**21), dict(x=A + 1), dict(gate=B + 1),
    dict(weight_dtype=F32, down=D + 2), dict(y=A + 1)], ids=str)
def test_forward_refusals(L, changes):
    assert refused(L, "gpga_feed_forward_forward", **changes)


def test_forward_of_no_tokens(L):
    nothing = {**FORWARD, **dict(rows=0, x=0, y=0, gate=0, up=0, down=0, scratch=0, scratch_bytes=0)}
    assert L.gpga_feed_forward_forward(packed("gpga_feed_forward_forward", nothing), None) == pkg.GPGA_OK


@pytest.mark.parametrize("changes", [
    dict(dy=0), dict(x=0), dict(g=0), dict(u=0), dict(gate=0), dict(up=0), dict(down=0), dict(dx=0), dict(dgate=0), dict(dup=0), dict(ddown=0),
    dict(scratch=0), dict(scratch=S + 4), dict(scratch_bytes=100), dict(lddy=d - 1), dict(ldx=d - 1), dict(ldg=f - 1), dict(ldu=f - 1), dict(lddx=d - 1),
    dict(ldgate=d - 1), dict(lddgate=d - 1), dict(lddup=d - 1), dict(ldddown=f - 1), dict(node_dgate=f * d - 1), dict(node_dup=0), dict(node_ddown=-1),
    dict(node_up=-1), dict(dtype=5), dict(weight_dtype=F16), dict(grad_dtype=F16), dict(grad_dtype=3), dict(activation=9), dict(nodes=0), dict(rows=2**31),
    dict(d=0), dict(f=0), dict(dgate=B + 2), dict(dy=A + 1), dict(rows=0, dgate=0)], ids=str)
def test_backward_refusals(L, changes):
    assert refused(L, "gpga_feed_forward_backward", **changes)


def test_backward_of_no_tokens_adds_nothing(L):
    nothing = {**BACKWARD, **dict(rows=0, dy=0, x=0, g=0, u=0, dx=0, gate=0, up=0, down=0, scratch=0, scratch_bytes=0, accumulate=1)}
    assert L.gpga_feed_forward_backward(packed("gpga_feed_forward_backward", nothing), None) == pkg.GPGA_OK


@pytest.mark.parametrize("changes", [
    dict(update=0), dict(out=0), dict(scratch=0), dict(scratch=S + 8), dict(scratch_bytes=0), dict(ldm=599), dict(ldo=599), dict(node_ldm=-1),
    dict(node_ldo=500 * 600 - 1), dict(node_ldo=0), dict(dtype=3), dict(nodes=0), dict(nodes=65536), dict(r=0), dict(c=0), dict(r=2**20 + 1),
    dict(c=2**20 + 1, ldm=2**21, ldo=2**21), dict(steps=0), dict(steps=1001), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(c1=float("nan")), dict(c3=float("inf")), dict(c5=float("-inf")), dict(scale=float("nan")), dict(update=A + 2), dict(out=B + 1)], ids=str)
def test_orthogonalize_refusals(L, changes):
    assert refused(L, "gpga_orthogonalize", **changes)


def scratch(L, name, **changes):
    return getattr(L, name + "_scratch_bytes")(packed(name, {**SAME_ROWS[name], **changes}))


def test_scratch_is_what_the_arguments_need(L):
    """Operands that a tiled copy can read where they lie take none; others their packed pieces of 16 bits."""
    big = dict(rows=100)
    h = n * 100 * f * 2
    assert h <= scratch(L, "gpga_feed_forward_forward", **big) < h + 256
    weights = 2 * n * f * d * 3 * 2                  # fp32 weights beside 16-bit activations: two pieces each
    assert h + weights <= scratch(L, "gpga_feed_forward_forward", weight_dtype=F32, **big) < h + weights + 4 * 256
    assert scratch(L, "gpga_feed_forward_forward", gate=B + 2, **big) >= h + n * f * d * 2
    pieces = 3 * 2 * (n * 100 * (d + f) + 3 * n * f * d)     # all fp32: three pieces each
    assert pieces <= scratch(L, "gpga_feed_forward_forward", dtype=F32, weight_dtype=F32, **big) < pieces + 5 * 256
    few = n * 8 * f
    assert scratch(L, "gpga_feed_forward_forward", rows=8) == few * 4          # h and the rests of its rounding
    assert scratch(L, "gpga_feed_forward_forward", rows=9) == n * 9 * f * 2
    assert scratch(L, "gpga_feed_forward_forward", rows=8, dtype=F32, weight_dtype=F32) == few * 4
    assert scratch(L, "gpga_feed_forward_forward", rows=0) == 0
    between = 3 * n * t * f * 2 + weights
    assert between <= scratch(L, "gpga_feed_forward_backward") < between + 6 * 256
    assert scratch(L, "gpga_orthogonalize") >= 2 * 2 * n * (2 * 500 * 600 + 2 * 500 * 500)
    assert scratch(L, "gpga_orthogonalize", r=100, c=300, ldm=300, ldo=300) == 0      # in one launch
    for name, wrong in (("gpga_feed_forward_forward", dict(d=0)), ("gpga_feed_forward_backward", dict(dtype=9)), ("gpga_orthogonalize", dict(steps=0))):
        assert scratch(L, name, **wrong) == 0


def test_binding_refuses_what_is_not_on_a_gpu():
    x, w, o = torch.ones(4, 8), torch.ones(16, 8), torch.ones(8, 16)
    for call in (lambda: pkg.feed_forward_forward(x, w, w, o), lambda: pkg.feed_forward_backward(x, x, x, x, w, w, o), lambda: pkg.orthogonalize(w),
                 lambda: pkg.orthogonalize(w.double()), lambda: pkg.feed_forward_forward(x, w.half(), w.half(), o.half())):
        with pytest.raises(pkg.GpgaError) as err:
            call()
        assert err.value.status == pkg.GPGA_ERR_INVALID_ARG


def test_matrix_arguments():
    """What the binding makes of a matrix per node (device -1 stands for the CPU's tensors here, which are refused)."""
    with pytest.raises(pkg.GpgaError):
        token_ops._matrix(torch.ones(3, 4), "w", (torch.float32,), -1)
    with pytest.raises(pkg.GpgaError):
        token_ops._activation("tanh")
    assert [token_ops._activation(a) for a in ("silu", "gelu", "relu")] == [0, 1, 2]


def code(name):
    """A source file without its comments."""
    text = (CSRC / name).read_text()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


@pytest.mark.parametrize("name", ["gpga_gemm.cuh", "gpga_gemm.cu", "gpga_pack.cuh", "gpga_ff_device.cuh", "gpga_ff_forward.cu", "gpga_ff_backward.cu",
                                  "gpga_ff_few.cu", "gpga_orth.cu", "gpga_matrix_api.cu"])
def test_host_statics_can_be_shared_by_threads(name):
    """What a host function keeps from one call to the next is initialised once by the language (const) or atomic."""
    kept = re.findall(r"^\s+static (?!__device__|inline\b|constexpr\b|cudaError_t\b)[^;({]*", code(name), flags=re.M)
    assert all(re.match(r"\s+static (const |std::atomic<)", s) for s in kept), kept


def test_copies_are_never_multicast():
    """Both blocks of a pair load their own halves; the arrival of finished products is all that goes to both."""
    text = "".join(code(p.name) for p in CSRC.glob("*.cu*"))
    for line in re.findall(r'"[^"]*multicast[^"]*"', text):
        assert "tcgen05.commit" in line, line


@pytest.mark.parametrize("k", [1, 63, 64, 65, 700])
def test_splits_of_a_sum_cover_it_once(k):
    """The parts of the k-blocks that the blocks of a cluster take (as the kernel computes them)."""
    blocks = -(-k // 64)
    for splits in (s for s in (1, 2, 4, 8) if s <= blocks):
        ends = [blocks * r // splits for r in range(splits + 1)]
        assert ends[0] == 0 and ends[-1] == blocks and all(a < b for a, b in zip(ends, ends[1:]))


def test_triangle_of_tiles_is_covered_once():
    """The tile of a symmetric product by its number: column j has j + 1 tiles (as the kernel computes them, in fp32)."""
    import numpy as np
    seen, r = set(), 0
    for j in range(60):
        for i in range(j + 1):
            got = int((np.sqrt(np.float32(8) * np.float32(r) + np.float32(1)) - np.float32(1)) * np.float32(0.5))
            while got * (got + 1) // 2 > r:
                got -= 1
            while (got + 1) * (got + 2) // 2 <= r:
                got += 1
            seen.add((r - got * (got + 1) // 2, got))
            assert (r - got * (got + 1) // 2, got) == (i, j)
            r += 1
    assert len(seen) == r
