"""Host-side checks of the token-block operators' C entries: arguments are judged before CUDA is touched, and the
binding packs the structs as a C compiler lays them out."""
import shutil
import subprocess
from pathlib import Path

import pytest

import paper_2105_09080_b200 as pkg
from paper_2105_09080_b200 import token_ops

A, B, S = 0x10000, 0x20000, 0x30000        # made-up aligned addresses, never read
F32, BF16 = 0, 1
MEMBERS = {
    "gpga_embedding_forward": "table tokens out ldt node_ldt ldo token_bytes dtype nodes rows d vocab scale",
    "gpga_embedding_backward": "dout tokens grad scratch scratch_bytes ldo ldg node_ldg token_bytes dtype nodes rows d vocab accumulate scale",
    "gpga_dropout": "x y ldx ldy dtype nodes rows d p seed k site node0",
    "gpga_layer_norm_forward": "x residual weight bias y z mean rstd ldx ldr ldw ldy ldz dtype nodes rows d eps p seed k site node0",
    "gpga_layer_norm_backward": "dy z dz mean rstd weight dresidual dx dweight dbias scratch scratch_bytes lddy ldz lddz ldw lddr lddx lddw "
                                "accumulate dtype nodes rows d p seed k site node0",
}


@pytest.fixture(scope="module")
def L():
    return pkg.lib()


def refused(L, st):
    return st == pkg.GPGA_ERR_INVALID_ARG and len(L.gpga_last_error(None)) > 0


def call(L, name, **values):
    return getattr(L, name)(token_ops.ARGS[name].pack(*(values[m] for m in MEMBERS[name].split())), None)


def test_structs_are_packed_as_in_c(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    lines = []
    for name, members in MEMBERS.items():
        for m in members.split():
            lines.append(f'printf("%zu ", offsetof({name}_args_t, {m}));')
        lines.append(f'printf("%zu\\n", sizeof({name}_args_t));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gpga.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-I", str(Path(__file__).resolve().parent.parent / "include"), str(src), "-o", str(tmp_path / "layout")],
                   check=True)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines()
    for (name, members), line in zip(MEMBERS.items(), out):
        n = len(members.split())
        assert [int(x) for x in line.split()] == [8 * i for i in range(n + 1)], name
        assert token_ops.ARGS[name].size == 8 * n
        assert getattr(pkg.lib(), name)(None, None) == pkg.GPGA_ERR_INVALID_ARG


def test_embedding_forward(L):
    def f(**kw):
        return call(L, "gpga_embedding_forward", **{**dict(table=A, ldt=16, node_ldt=9 * 16, tokens=B, token_bytes=8, out=S, ldo=16, dtype=F32, nodes=2,
                                                           rows=3, d=16, vocab=9, scale=1.0), **kw})
    for kw in (dict(table=0), dict(tokens=0), dict(out=0), dict(ldt=15), dict(ldo=15), dict(token_bytes=2), dict(dtype=3), dict(dtype=-1),
               dict(dtype=2**32), dict(nodes=0), dict(nodes=65536), dict(rows=-1), dict(rows=2**31), dict(d=0),
               dict(d=2**20 + 1, ldt=2**21, ldo=2**21), dict(vocab=0), dict(vocab=2**31), dict(table=A + 2), dict(tokens=B + 4), dict(out=S + 2),
               dict(dtype=BF16, out=S + 1)):
        assert refused(L, f(**kw)), kw
    assert f(rows=0) == pkg.GPGA_OK
    assert f(rows=0, table=0, tokens=0, out=0) == pkg.GPGA_OK


def test_embedding_backward(L):
    need = L.gpga_embedding_scratch_bytes(2, 3000, 16, 9)
    assert need > 0 and L.gpga_embedding_scratch_bytes(2, 3, 16, 9) == 0     # few tokens take no scratch

    def f(**kw):
        return call(L, "gpga_embedding_backward", **{**dict(dout=A, ldo=16, dtype=F32, tokens=B, token_bytes=4, grad=S, ldg=16, node_ldg=9 * 16,
                                                            nodes=2, rows=3000, d=16, vocab=9, accumulate=0, scratch=0x40000, scratch_bytes=need,
                                                            scale=1.0), **kw})
    for kw in (dict(dout=0), dict(tokens=0), dict(grad=0), dict(scratch=0), dict(scratch=0x40008), dict(scratch_bytes=need - 1), dict(ldg=15),
               dict(node_ldg=9 * 16 - 1), dict(ldo=8), dict(dtype=5), dict(token_bytes=1), dict(vocab=0), dict(nodes=0), dict(d=0)):
        assert refused(L, f(**kw)), kw
    assert f(rows=0, accumulate=1) == pkg.GPGA_OK            # nothing to add, nothing launched
    assert L.gpga_embedding_scratch_bytes(0, 3, 16, 9) == 0
    # the scratch area does not grow with what one call sorts at a time
    assert L.gpga_embedding_scratch_bytes(1, 65536, 64, 1000) == L.gpga_embedding_scratch_bytes(1, 10**6, 64, 1000)


def test_dropout(L):
    def f(**kw):
        return call(L, "gpga_dropout", **{**dict(x=A, ldx=16, y=B, ldy=16, dtype=F32, nodes=2, rows=3, d=16, p=0.5, seed=1, k=0, site=0, node0=0), **kw})
    for kw in (dict(x=0), dict(y=0), dict(ldx=1), dict(ldy=15), dict(dtype=9), dict(p=-0.1), dict(p=1.01), dict(p=float("nan")), dict(k=-1),
               dict(k=2**32), dict(site=-1), dict(site=2**30), dict(node0=-1), dict(node0=2**32 - 1), dict(x=A + 1),
               dict(rows=2**30, d=64, ldx=64, ldy=64), dict(nodes=2**15, rows=2**16)):
        assert refused(L, f(**kw)), kw
    assert f(rows=0) == pkg.GPGA_OK


def test_layer_norm(L):
    def fwd(**kw):
        return call(L, "gpga_layer_norm_forward", **{**dict(x=A, ldx=16, residual=0, ldr=0, weight=S, bias=S, ldw=16, y=B, ldy=16, z=0, ldz=0,
                                                            mean=0x50000, rstd=0x60000, dtype=F32, nodes=2, rows=3, d=16, eps=1e-5, p=0.0, seed=1, k=0,
                                                            site=0, node0=0), **kw})
    for kw in (dict(x=0), dict(y=0), dict(mean=0), dict(rstd=0), dict(ldx=8), dict(ldy=8), dict(residual=A, ldr=8), dict(z=A, ldz=8), dict(ldw=-1),
               dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e300), dict(p=2.0), dict(p=0.5, k=-1), dict(d=0),
               dict(dtype=7), dict(weight=S + 2), dict(mean=0x50002)):
        assert refused(L, fwd(**kw)), kw
    assert fwd(rows=0) == pkg.GPGA_OK

    need = L.gpga_layer_norm_scratch_bytes(2, 3000, 16)
    assert need > 0 and L.gpga_layer_norm_scratch_bytes(2, 3000, 0) == 0

    def bwd(**kw):
        return call(L, "gpga_layer_norm_backward", **{**dict(dy=A, lddy=16, z=B, ldz=16, dz=0, lddz=0, mean=0x50000, rstd=0x60000, weight=S, ldw=16,
                                                             dresidual=0x70000, lddr=16, dx=0, lddx=0, dweight=0x80000, dbias=0x90000, lddw=16,
                                                             accumulate=0, dtype=F32, nodes=2, rows=3000, d=16, p=0.0, seed=1, k=0, site=0, node0=0,
                                                             scratch=0x100000, scratch_bytes=need), **kw})
    for kw in (dict(dy=0), dict(z=0), dict(mean=0), dict(rstd=0), dict(dresidual=0), dict(lddy=1), dict(ldz=1), dict(dz=A, lddz=1),
               dict(lddr=1), dict(lddw=15), dict(p=0.5), dict(p=0.0, dx=A, lddx=16), dict(p=0.5, dx=A, lddx=3), dict(scratch=0),
               dict(scratch=0x100004), dict(scratch_bytes=need - 1), dict(dtype=4), dict(nodes=0)):
        assert refused(L, bwd(**kw)), kw
