"""Host-side checks (CPU) of the embedding, residual norm and clipping calls: workspace sizes, and bad arguments that the C
entry points refuse before any launch."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1905_07931_amd", "libl1csr.so")
OK, EINVAL, EUNSUPPORTED = 0, -1, -5
OP_PLAN, OP_BWD, OP_NORM, OP_CLIP = 17, 18, 19, 20
NO_GPU = not os.path.exists("/dev/kfd")
BIG = 1 << 40
nan, inf = float("nan"), float("inf")
pytestmark = pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")


def at(i, off=0):  # far apart, never dereferenced
    return C.c_void_p((1 << 44) + (i << 38) + off)


@pytest.fixture(scope="module")
def lib():
    import paper_1905_07931_amd as L1
    if not os.path.exists(LIB):
        from paper_1905_07931_amd import build
        build.build(verbose=False)
    return L1.lib()


def test_workspace_sizes(lib):
    ws = lib.l1csr_workspace_bytes
    for B in (1, 64, 8192, 8193, 1 << 24):
        assert ws(OP_PLAN, 100, 0, 0, B) >= 12 * B
        assert ws(OP_BWD, 100, 10, 0, B) >= 40 * B
        assert ws(OP_NORM, 100, 0, 0, B) > 0
    assert ws(OP_PLAN, 100, 0, 0, (1 << 24) + 1) == 0 and ws(OP_BWD, 100, 10, 0, (1 << 24) + 1) == 0
    assert ws(OP_BWD, 100, 0, 0, 5) == 0 and ws(OP_BWD, 0, 5, 0, 5) == 0 and ws(OP_NORM, 0, 0, 0, 5) == 0
    assert ws(OP_NORM, (1 << 24) + 1, 0, 0, 4) == 0
    assert 0 < ws(OP_CLIP, 1, 0, 0, 0) <= ws(OP_CLIP, 1000, 0, 0, 0)


def lookup(lib, V=8, D=8, B=8, dtype=0, E=at(0), lde=8, tokens=at(1), scale=1.0, xd=0, X=at(2), ldx=8):
    return lib.l1csr_embedding_fwd(V, D, B, dtype, E, lde, tokens, scale, xd, X, ldx, None)


def lookup_csr(lib, V=8, D=8, nnz=9, ptr=at(3), idx=at(4), vals=at(5), B=8, tokens=at(1), scale=1.0, X=at(2), ldx=8):
    return lib.l1csr_embedding_csr_fwd(V, D, nnz, ptr, idx, vals, B, tokens, scale, X, ldx, None)


def plan(lib, V=8, B=8, tokens=at(1), p=at(6), n=BIG):
    return lib.l1csr_embedding_plan(V, B, tokens, p, n, None)


def bwd(lib, V=8, D=8, B=8, dtype=0, dX=at(2), ldx=8, p=at(6), pn=BIG, scale=1.0, ed=0, add=None, lda=8, dE=at(0), lde=8,
        ws=at(7), n=BIG):
    return lib.l1csr_embedding_bwd(V, D, B, dtype, dX, ldx, p, pn, scale, ed, add, lda, dE, lde, ws, n, None)


def masked(lib, V=8, D=8, nnz=9, ptr=at(3), idx=at(4), B=8, dX=at(2), ldx=8, p=at(6), pn=BIG, scale=1.0, gv=at(5), ws=at(7), n=BIG):
    return lib.l1csr_embedding_masked_bwd(V, D, nnz, ptr, idx, B, dX, ldx, p, pn, scale, gv, ws, n, None)


def test_embedding_arguments(lib):
    many = (1 << 24) + 1
    for kw in (dict(V=-1), dict(D=-1), dict(B=-1), dict(dtype=3), dict(dtype=1, xd=2), dict(E=None), dict(lde=7), dict(tokens=None),
               dict(scale=nan), dict(scale=inf), dict(X=None), dict(ldx=7), dict(X=at(0)), dict(X=at(1)), dict(X=at(0, 100)),
               dict(xd=1)):
        assert lookup(lib, **kw) == EINVAL, kw
    assert lookup(lib, B=many, ldx=many) == EUNSUPPORTED and lookup(lib, V=(1 << 30) + 1) == EUNSUPPORTED
    for kw in (dict(nnz=-1), dict(nnz=65), dict(ptr=None), dict(idx=None), dict(vals=None), dict(tokens=None), dict(X=None),
               dict(ldx=7), dict(scale=nan), dict(X=at(1)), dict(X=at(3)), dict(X=at(4)), dict(X=at(5)), dict(B=-1)):
        assert lookup_csr(lib, **kw) == EINVAL, kw
    for kw in (dict(V=-1), dict(B=-1), dict(tokens=None), dict(p=None), dict(n=95), dict(p=at(1)), dict(p=at(6, 2))):
        assert plan(lib, **kw) == EINVAL, kw
    assert plan(lib, B=many) == EUNSUPPORTED and plan(lib, B=0, tokens=None, p=None, n=0) == OK
    for kw in (dict(V=-1), dict(D=-1), dict(B=-1), dict(dtype=3), dict(dtype=1, ed=2), dict(ed=1), dict(dX=None), dict(ldx=7),
               dict(p=None), dict(pn=95), dict(scale=inf), dict(dE=None), dict(lde=7), dict(add=at(8), lda=7),
               dict(add=at(0), lda=9), dict(add=at(0, 4)), dict(dE=at(2)), dict(dE=at(6)), dict(ws=None), dict(n=100),
               dict(ws=at(7, 8))):
        assert bwd(lib, **kw) == EINVAL, kw
    assert bwd(lib, B=many, ldx=many) == EUNSUPPORTED
    assert bwd(lib, V=0, dE=None) == OK and bwd(lib, D=0, dX=None, dE=None, ws=None, n=0) == OK
    for kw in (dict(nnz=-1), dict(nnz=65), dict(ptr=None), dict(idx=None), dict(dX=None), dict(ldx=7), dict(p=None), dict(gv=None),
               dict(gv=at(2)), dict(gv=at(3)), dict(gv=at(4)), dict(gv=at(6)), dict(ws=None), dict(n=100), dict(scale=nan)):
        assert masked(lib, **kw) == EINVAL, kw


def fwd_norm(lib, K=8, B=8, dtype=0, r=at(0), ldr=8, y=at(1), ldy=8, kind=2, sig=0, gate=at(2), ldg=8, post=at(3), pre=at(4),
             alpha=1.0, eps=1e-6, ro=at(5), ldro=8, h=at(6), ldh=8, ws=at(7), n=BIG):
    return lib.l1csr_residual_norm_fwd(K, B, dtype, r, ldr, y, ldy, kind, sig, gate, ldg, post, pre, alpha, eps, ro, ldro, h, ldh,
                                       ws, n, None)


def bwd_norm(lib, K=8, B=8, dtype=0, r=at(0), ldr=8, dro=at(1), lddro=8, dh=at(2), lddh=8, y=at(3), ldy=8, kind=2, sig=0, gate=at(4),
             ldg=8, post=at(5), pre=at(6), alpha=1.0, eps=1e-6, dr=at(7), lddr=8, dy=at(8), lddy=8, dg=at(9), lddg=8, dpost=at(10),
             dpre=at(11), ws=at(12), n=BIG):
    return lib.l1csr_residual_norm_bwd(K, B, dtype, r, ldr, dro, lddro, dh, lddh, y, ldy, kind, sig, gate, ldg, post, pre, alpha,
                                       eps, dr, lddr, dy, lddy, dg, lddg, dpost, dpre, ws, n, None)


def test_norm_arguments(lib):
    for kw in (dict(K=-1), dict(B=-1), dict(dtype=3), dict(r=None), dict(ldr=7), dict(ldy=7), dict(kind=3), dict(kind=-1),
               dict(gate=None), dict(ldg=7), dict(alpha=nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=inf), dict(ro=None),
               dict(ldro=7), dict(h=None), dict(ldh=7), dict(pre=None), dict(y=None), dict(ws=None), dict(n=10), dict(ws=at(7, 8)),
               dict(ro=at(2)), dict(h=at(5)), dict(h=at(2)), dict(ro=at(3)), dict(h=at(4)), dict(ro=at(0), ldro=9),
               dict(ro=at(0, 4)), dict(kind=1, ro=at(2)), dict(y=None, kind=0, post=None)):
        assert fwd_norm(lib, **kw) == EINVAL, kw
    assert fwd_norm(lib, K=(1 << 24) + 1) == EUNSUPPORTED
    for kw in (dict(K=-1), dict(dtype=4), dict(r=None), dict(dh=None), dict(dr=None), dict(dy=None), dict(dg=None), dict(dpre=None),
               dict(dpost=None), dict(post=None), dict(pre=None), dict(kind=0), dict(kind=1, dg=None), dict(ldr=7), dict(lddro=7),
               dict(lddh=7), dict(lddr=7), dict(lddy=7), dict(lddg=7), dict(eps=0.0), dict(dr=at(0)), dict(dr=at(3)),
               dict(dy=at(2)), dict(dy=at(1)), dict(dg=at(3)), dict(dr=at(8)), dict(dpre=at(0)), dict(dpre=at(5)),
               dict(dpost=at(11)), dict(dpre=at(7)), dict(dr=at(1), lddr=9), dict(dy=at(3, 4)), dict(n=10), dict(ws=None)):
        assert bwd_norm(lib, **kw) == EINVAL, kw
    assert bwd_norm(lib, B=(1 << 24) + 1, **{k: 1 << 25 for k in ("ldr", "lddro", "lddh", "ldy", "ldg", "lddr", "lddy", "lddg")}) == EUNSUPPORTED


def clip(lib, g=(at(0), at(1)), rows=(4, 1), cols=(5, 9), ld=(6, 9), dt=(0, 1), out=None, ldo=None, odt=None, max_norm=1.0,
         scale=1.0, eps=1e-6, zero=0, stats=at(9), ws=at(10), n=BIG, count=None):
    k = len(g)
    vp = lambda x: None if x is None else (C.c_void_p * k)(*[p.value for p in x])  # noqa: E731
    i64 = lambda x: None if x is None else (C.c_int64 * k)(*x)  # noqa: E731
    i32 = lambda x: None if x is None else (C.c_int32 * k)(*x)  # noqa: E731
    return lib.l1csr_clip_grad_norm(k if count is None else count, vp(g), i64(rows), i64(cols), i64(ld), i32(dt), vp(out), i64(ldo),
                                    i32(odt), max_norm, scale, eps, zero, stats, ws, n, None)


def test_clip_arguments(lib):
    for kw in (dict(count=-1), dict(g=(at(0), C.c_void_p(0))), dict(rows=(-1, 1)), dict(cols=(5, -1)), dict(ld=(4, 9)), dict(dt=(3, 0)),
               dict(max_norm=-1.0), dict(max_norm=nan), dict(scale=0.0), dict(scale=-1.0), dict(scale=inf), dict(eps=0.0),
               dict(eps=nan), dict(stats=None), dict(stats=at(0)), dict(stats=at(1, 8)), dict(ws=None), dict(n=100), dict(ws=at(10, 8)),
               dict(g=(at(0), at(0))), dict(g=(at(0), at(0, 44))), dict(out=(at(2), at(2))), dict(out=(at(1), at(0))),
               dict(out=(at(2), at(3)), ldo=(4, 9)), dict(out=(at(2), at(3)), odt=(1, 1)), dict(out=(at(0), at(3)), ldo=(7, 9)),
               dict(out=(at(0, 4), at(3)), ldo=(6, 9)), dict(out=(at(2), at(1)), odt=(0, 0)),
               dict(out=(at(2), at(2, 79)), odt=(0, 1))):
        assert clip(lib, **kw) == EINVAL, kw
    assert clip(lib, rows=(1 << 31, 1)) == EUNSUPPORTED
    args = [(C.c_void_p * 1)(at(0).value), (C.c_int64 * 1)(1), (C.c_int64 * 1)(5), (C.c_int64 * 1)(5), (C.c_int32 * 1)(0)]
    for i in range(5):
        assert lib.l1csr_grad_norm(1, *[None if j == i else x for j, x in enumerate(args)], 1.0, at(9), at(10), BIG, None) == EINVAL
    assert lib.l1csr_grad_norm(1, *args, 0.0, at(9), at(10), BIG, None) == EINVAL
    assert lib.l1csr_grad_norm(1, *args, 1.0, None, at(10), BIG, None) == EINVAL
