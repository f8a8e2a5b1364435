"""Host-side checks of the token-block operators' C entries: arguments are judged before CUDA is touched."""
import pytest

import paper_2105_09080_b200 as pkg

A, B, S = 0x10000, 0x20000, 0x30000        # made-up aligned addresses, never read
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def L():
    return pkg.lib()


def refused(L, st):
    return st == pkg.GPGA_ERR_INVALID_ARG and len(L.gpga_last_error(None)) > 0


def test_embedding_forward(L):
    def call(table=A, ldt=16, tokens=B, tb=8, out=S, ldo=16, dtype=F32, nodes=2, rows=3, d=16, vocab=9):
        return L.gpga_embedding_forward(table, ldt, 9 * 16, tokens, tb, out, ldo, dtype, nodes, rows, d, vocab, 1.0, None)
    for kw in (dict(table=None), dict(tokens=None), dict(out=None), dict(ldt=15), dict(ldo=15), dict(tb=2), dict(dtype=3), dict(dtype=-1),
               dict(nodes=0), dict(nodes=65536), dict(rows=-1), dict(rows=2**31), dict(d=0), dict(d=2**20 + 1, ldt=2**21, ldo=2**21),
               dict(vocab=0), dict(vocab=2**31), dict(table=A + 2), dict(tokens=B + 4), dict(out=S + 2), dict(dtype=BF16, out=S + 1)):
        assert refused(L, call(**kw)), kw
    assert call(rows=0) == pkg.GPGA_OK
    assert call(rows=0, table=None, tokens=None, out=None) == pkg.GPGA_OK


def test_embedding_backward(L):
    need = L.gpga_embedding_scratch_bytes(2, 3, 16, 9)
    assert need > 0

    def call(dout=A, ldo=16, dtype=F32, tokens=B, tb=4, grad=S, ldg=16, node_ldg=9 * 16, nodes=2, rows=3, d=16, vocab=9, acc=0,
             scratch=0x40000, nbytes=need):
        return L.gpga_embedding_backward(dout, ldo, dtype, tokens, tb, grad, ldg, node_ldg, nodes, rows, d, vocab, 1.0, acc, scratch, nbytes,
                                         None)
    for kw in (dict(dout=None), dict(tokens=None), dict(grad=None), dict(scratch=None), dict(scratch=0x40008), dict(nbytes=need - 1),
               dict(ldg=15), dict(node_ldg=9 * 16 - 1), dict(ldo=8), dict(dtype=5), dict(tb=1), dict(vocab=0), dict(nodes=0), dict(d=0)):
        assert refused(L, call(**kw)), kw
    assert call(rows=0, acc=1) == pkg.GPGA_OK            # nothing to add, nothing launched
    assert L.gpga_embedding_scratch_bytes(0, 3, 16, 9) == 0
    # the scratch area does not grow with what one call sorts at a time
    assert L.gpga_embedding_scratch_bytes(1, 65536, 64, 1000) == L.gpga_embedding_scratch_bytes(1, 10**6, 64, 1000)


def test_dropout(L):
    def call(x=A, ldx=16, y=B, ldy=16, dtype=F32, nodes=2, rows=3, d=16, p=0.5, k=0, site=0, node0=0):
        return L.gpga_dropout(x, ldx, y, ldy, dtype, nodes, rows, d, p, 1, k, site, node0, None)
    for kw in (dict(x=None), dict(y=None), dict(ldx=1), dict(ldy=15), dict(dtype=9), dict(p=-0.1), dict(p=1.01), dict(p=float("nan")),
               dict(k=-1), dict(k=2**32), dict(site=-1), dict(site=2**30), dict(node0=-1), dict(node0=2**32 - 1), dict(x=A + 1),
               dict(rows=2**30, d=64, ldx=64, ldy=64), dict(nodes=2**15, rows=2**16)):
        assert refused(L, call(**kw)), kw
    assert call(rows=0) == pkg.GPGA_OK


def test_layer_norm(L):
    def fwd(x=A, ldx=16, r=None, ldr=0, w=S, b=S, ldw=16, y=B, ldy=16, z=None, ldz=0, mean=0x50000, rstd=0x60000, dtype=F32, nodes=2, rows=3,
            d=16, eps=1e-5, p=0.0, k=0):
        return L.gpga_layer_norm_forward(x, ldx, r, ldr, w, b, ldw, y, ldy, z, ldz, mean, rstd, dtype, nodes, rows, d, eps, p, 1, k, 0, 0, None)
    for kw in (dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(ldx=8), dict(ldy=8), dict(r=A, ldr=8), dict(z=A, ldz=8),
               dict(ldw=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(p=2.0), dict(p=0.5, k=-1), dict(d=0),
               dict(dtype=7), dict(w=S + 2), dict(mean=0x50002)):
        assert refused(L, fwd(**kw)), kw
    assert fwd(rows=0) == pkg.GPGA_OK

    need = L.gpga_layer_norm_scratch_bytes(2, 3000, 16)
    assert need > 0 and L.gpga_layer_norm_scratch_bytes(2, 3000, 0) == 0

    def bwd(dy=A, lddy=16, z=B, ldz=16, dz=None, lddz=0, mean=0x50000, rstd=0x60000, w=S, ldw=16, dres=0x70000, lddr=16, dx=None, lddx=0,
            dw=0x80000, db=0x90000, lddw=16, dtype=F32, nodes=2, rows=3000, d=16, p=0.0, scratch=0x100000, nbytes=need):
        return L.gpga_layer_norm_backward(dy, lddy, z, ldz, dz, lddz, mean, rstd, w, ldw, dres, lddr, dx, lddx, dw, db, lddw, 0, dtype, nodes,
                                          rows, d, p, 1, 0, 0, 0, scratch, nbytes, None)
    for kw in (dict(dy=None), dict(z=None), dict(mean=None), dict(rstd=None), dict(dres=None), dict(lddy=1), dict(ldz=1), dict(dz=A, lddz=1),
               dict(lddr=1), dict(lddw=15), dict(p=0.5), dict(p=0.0, dx=A, lddx=16), dict(p=0.5, dx=A, lddx=3), dict(scratch=None),
               dict(scratch=0x100004), dict(nbytes=need - 1), dict(dtype=4), dict(nodes=0)):
        assert refused(L, bwd(**kw)), kw
