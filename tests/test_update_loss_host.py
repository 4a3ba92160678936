"""Host-side checks (CPU) of muon_update and the losses over logits: workspace sizes, and bad arguments that the C entry
points refuse before any launch; the binding's own checks of tensors."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1905_07931_amd", "libl1csr.so")
OK, EINVAL, EUNSUPPORTED = 0, -1, -5
OP_MUON, OP_MUON_F16, OP_TOKEN_LOSS = 14, 15, 16
NO_GPU = not os.path.exists("/dev/kfd")
P, Q, R, W = (C.c_void_p(1 << 20), C.c_void_p(1 << 30), C.c_void_p(1 << 33), C.c_void_p(1 << 36))  # never dereferenced
BIG = 1 << 40
nan, inf = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    import paper_1905_07931_amd as L1
    if not os.path.exists(LIB):
        from paper_1905_07931_amd import build
        build.build(verbose=False)
    return L1.lib()


def test_workspace_sizes(lib):
    ws = lib.l1csr_workspace_bytes
    for n, k in [(1, 1), (100, 300), (129, 129), (4096, 9216), (46340, 46340)]:
        for op in (OP_MUON, OP_MUON_F16):
            b = ws(op, n, k, 0, 0)
            assert b > 0 and b % 256 == 0 and b == ws(op, k, n, 0, 0)
        assert ws(OP_MUON, n, k, 0, 0) >= ws(OP_MUON_F16, n, k, 0, 0)
    assert ws(OP_MUON, 0, 5, 0, 0) == 0 and ws(OP_MUON, 5, 0, 0, 0) == 0 and ws(OP_MUON, -1, 5, 0, 0) == 0
    for c, b in [(1, 1), (10, 128), (131072, 7), (32768, 8192), (1, 1 << 20)]:
        n = ws(OP_TOKEN_LOSS, c, 0, 0, b)
        assert n % 256 == 0 and n >= 16 * b
        assert ws(OP_TOKEN_LOSS, c, 1000, 0, b) >= n + 8 * 900
    assert ws(OP_TOKEN_LOSS, 0, 0, 0, 5) == 0


def muon(lib, N=8, K=8, dtype=0, G=P, ldg=8, M=Q, ldm=8, M_out=Q, ldmo=8, mu=0.9, nesterov=1, steps=5, eps=1e-7, scale=1.0,
         precision=0, O=R, ldo=8, ws=W, ws_bytes=BIG):
    return lib.muon_update(N, K, dtype, G, ldg, M, ldm, M_out, ldmo, mu, nesterov, steps, eps, scale, precision, O, ldo, ws,
                           ws_bytes, None)


@pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")
def test_muon_arguments_are_rejected_before_launch(lib):
    bad = [dict(N=-1), dict(K=-1), dict(dtype=3), dict(dtype=-1), dict(precision=1), dict(precision=2), dict(precision=4),
           dict(steps=0), dict(steps=33), dict(eps=-1e-9), dict(eps=nan), dict(eps=inf), dict(scale=nan), dict(scale=inf),
           dict(mu=1.0), dict(mu=-0.1), dict(mu=nan), dict(G=None), dict(O=None), dict(ldg=7), dict(ldo=7), dict(ldm=7),
           dict(ldmo=7), dict(M=None), dict(ws=None), dict(ws_bytes=1000),
           dict(O=C.c_void_p((1 << 20) + 4)), dict(O=P, ldo=9), dict(M=P), dict(M_out=P), dict(M_out=R), dict(M=R),
           dict(M_out=C.c_void_p((1 << 30) + 4)), dict(ldmo=9)]
    for kw in bad:
        assert muon(lib, **kw) == EINVAL, kw
    big = dict(ldg=1 << 23, ldm=1 << 23, ldmo=1 << 23, ldo=1 << 23, M=None, M_out=None)
    assert muon(lib, N=1, K=(1 << 22) + 1, **big) == EUNSUPPORTED
    assert muon(lib, N=65536, K=32768, M=None, M_out=None, ldg=32768, ldo=32768, O=C.c_void_p(1 << 44)) == EUNSUPPORTED
    for n, k in ((0, 8), (8, 0), (0, 0)):  # nothing to do
        assert muon(lib, N=n, K=k, ws=None, ws_bytes=0) == OK


def policy(lib, Cn=8, B=8, dtype=0, z=P, ld=8, labels=Q, old=Q, adv=Q, ref=None, w=None, lo=0.2, hi=0.2, kl=0.1, dz=R,
           ldd=8, logp=None, stats=Q, ws=W, ws_bytes=BIG):
    return lib.l1csr_policy_loss(Cn, B, dtype, z, ld, labels, old, adv, ref, w, lo, hi, kl, dz, ldd, logp, stats, ws, ws_bytes,
                                 None)


def preference(lib, Cn=8, B=8, dtype=0, z=P, ld=8, labels=Q, pairs=2, ptr=Q, ref=None, w=None, beta=0.1, ls=0.0, dz=R, ldd=8,
               rewards=None, loss=Q, ws=W, ws_bytes=BIG):
    return lib.l1csr_preference_loss(Cn, B, dtype, z, ld, labels, pairs, ptr, ref, w, beta, ls, dz, ldd, rewards, loss, ws,
                                     ws_bytes, None)


@pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")
def test_loss_arguments_are_rejected_before_launch(lib):
    common = [dict(Cn=0), dict(Cn=-1), dict(B=-1), dict(dtype=3), dict(z=None), dict(ld=7), dict(ldd=7), dict(labels=None),
              dict(ws=None), dict(ws_bytes=100), dict(dz=C.c_void_p((1 << 20) + 4)), dict(dz=P, ldd=9)]
    for kw in common + [dict(old=None), dict(adv=None), dict(stats=None), dict(lo=-0.1), dict(lo=1.1), dict(lo=nan),
                        dict(hi=-0.1), dict(hi=inf), dict(kl=-0.1), dict(kl=nan)]:
        assert policy(lib, **kw) == EINVAL, kw
    for kw in common + [dict(pairs=-1), dict(ptr=None), dict(loss=None), dict(beta=-1.0), dict(beta=nan), dict(ls=-0.1),
                        dict(ls=0.6), dict(ls=nan), dict(pairs=(1 << 30))]:
        assert preference(lib, **kw) == EINVAL, kw
    logp = lambda **k: lib.l1csr_token_logp(*(k.get(n, d) for n, d in (  # noqa: E731
        ("Cn", 8), ("B", 8), ("dtype", 0), ("z", P), ("ld", 8), ("labels", Q), ("logp", R), ("ws", W), ("ws_bytes", BIG))), None)
    for kw in [dict(Cn=0), dict(B=-1), dict(dtype=7), dict(z=None), dict(ld=7), dict(labels=None), dict(logp=None),
               dict(ws=None), dict(ws_bytes=10)]:
        assert logp(**kw) == EINVAL, kw
    assert logp(B=0, logp=None, labels=None, ws=None, ws_bytes=0, z=None) == OK


@pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")
def test_outputs_of_the_losses_apart_from_their_inputs(lib):
    at = lambda i, off=0: C.c_void_p((1 << 44) + (i << 38) + off)  # noqa: E731
    z, labels, old, adv, ref, w, dz, logp, stats, ptr = (at(i) for i in range(10))
    good = dict(z=z, labels=labels, old=old, adv=adv, ref=ref, w=w, dz=dz, logp=logp, stats=stats)
    # (refused for their size only after every other check: what is left of the call is sound)
    assert policy(lib, **good, ws_bytes=0) == EINVAL and policy(lib, **good, Cn=(1 << 30) + 1) == EUNSUPPORTED
    for name, p in list(good.items()):
        for out in ("logp", "stats", "dz"):
            if out == name or (name, out) == ("z", "dz"):
                continue
            assert policy(lib, **{**good, out: p}) == EINVAL, (name, out)
    assert policy(lib, **{**good, "logp": at(2, 28)}) == EINVAL
    both = dict(z=z, labels=labels, ptr=ptr, ref=ref, w=w, dz=dz, rewards=logp, loss=stats)
    for name, p in list(both.items()):
        for out in ("rewards", "loss", "dz"):
            if out == name or (name, out) == ("z", "dz"):
                continue
            assert preference(lib, **{**both, out: p}) == EINVAL, (name, out)
    for p in (z, labels):
        assert lib.l1csr_token_logp(8, 8, 0, z, 8, labels, p, at(11), BIG, None) == EINVAL


@pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")
def test_sizes_past_the_kernels_numbers_are_refused(lib):
    many = (1 << 30) + 1
    assert policy(lib, Cn=many) == EUNSUPPORTED and policy(lib, B=many, ld=many, ldd=many) == EUNSUPPORTED
    assert preference(lib, Cn=many) == EUNSUPPORTED and preference(lib, pairs=1 << 24) == EUNSUPPORTED
    assert lib.l1csr_token_logp(many, 1, 2, P, 1, Q, R, W, BIG, None) == EUNSUPPORTED
    ws = lib.l1csr_workspace_bytes  # nothing to allocate for a call that is refused
    assert ws(OP_TOKEN_LOSS, many, 0, 0, 1) == 0 and ws(OP_TOKEN_LOSS, 8, 1 << 24, 0, 8) == 0
    assert ws(OP_MUON, 65536, 32768, 0, 0) == 0 and ws(OP_MUON_F16, (1 << 22) + 1, 1, 0, 0) == 0
    assert muon(lib, N=65536, K=32768, M=None, M_out=None, ldg=32768, ldo=32768, O=C.c_void_p(1 << 44), ws=None,
                ws_bytes=0) == EUNSUPPORTED


@pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")
def test_misaligned_workspaces_are_refused(lib):
    odd = C.c_void_p((1 << 36) + 8)
    far = dict(dz=C.c_void_p(1 << 40))
    assert muon(lib, ws=odd) == EINVAL
    assert policy(lib, stats=C.c_void_p(1 << 41), ws=odd, **far) == EINVAL
    assert preference(lib, loss=C.c_void_p(1 << 41), ws=odd, **far) == EINVAL
    assert lib.l1csr_token_logp(8, 8, 0, P, 8, Q, R, odd, BIG, None) == EINVAL


def test_binding_refuses_host_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    import paper_1905_07931_amd as L1
    z, lab = torch.zeros(4, 3), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        L1.token_logp(z, lab)
    with pytest.raises(ValueError):
        L1.policy_loss(z, lab, z[0], z[0])
    with pytest.raises(ValueError):
        L1.preference_loss(z, lab, lab)
    with pytest.raises(TypeError):
        L1.token_logp([[0.0]], lab)
    with pytest.raises(ValueError):
        L1.orthogonalize(z)
    with pytest.raises(TypeError):
        L1.orthogonalize(z.numpy())
    W = L1.CSR(4, 3, torch.zeros(5, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1), 0)
    for f in (L1.prox_muon_step, L1.prox_muon_recompress):
        with pytest.raises(ValueError):
            f(W, z, L1.MuonState(torch.zeros(4, 3)), 0.1, 0.1)
    for name in ("token_logp", "policy_loss", "preference_loss", "orthogonalize", "MuonState", "prox_muon_step",
                 "prox_muon_recompress", "F16"):
        assert name in L1.__all__ and hasattr(L1, name)


def test_workspaces_under_capture_are_not_the_streams(monkeypatch):
    """Scratch that a captured call uses stays out of the stream's cache, and the cache's buffer out of the graph."""
    torch = pytest.importorskip("torch")
    import paper_1905_07931_amd as L1
    capturing = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    monkeypatch.setattr(L1, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(L1, "_empty_bytes", lambda n, device, stream: torch.empty(n, dtype=torch.uint8))
    monkeypatch.setattr(L1, "_ws_cache", {})
    dev = torch.device("cuda", 0)
    eager, n = L1._workspace(1000, dev)
    assert n == 1000 and L1._workspace(500, dev)[0] is eager
    capturing[0] = True
    first, second = L1._workspace(500, dev)[0], L1._workspace(2000, dev)[0]
    assert first is not eager and first.numel() == 500 and second.numel() == 2000
    assert list(L1._ws_cache.values()) == [eager]
    capturing[0] = False
    assert L1._workspace(1000, dev)[0] is eager


def test_prox_muon_refuses_to_write_into_what_it_reads():
    """The check of the Prox-Muon calls' written tensors against the layer's arrays, on host tensors."""
    torch = pytest.importorskip("torch")
    import paper_1905_07931_amd as L1
    N, K = 4, 6
    full = lambda: L1.CSR(N, K, torch.arange(0, N * K + 1, K, dtype=torch.int32),  # noqa: E731
                          torch.arange(K, dtype=torch.int32).repeat(N), torch.ones(N * K), N * K)
    W, st = full(), L1.MuonState(torch.zeros(N, K))
    Z, new, counts = torch.zeros(N, K), torch.zeros(N, K), torch.zeros(N, dtype=torch.int32)
    wide = torch.zeros(N, 2 * K)
    L1._muon_writes(W, Z, st)
    L1._muon_writes(W, Z, st, new, counts)
    L1._muon_writes(W, wide[:, :K], L1.MuonState(wide[:, K:]), new, counts)  # columns of one buffer
    over = W.vals.view(N, K)
    cols = W.col_idx.view(torch.float32).view(N, K)
    bad = [(over, st, None, None), (cols, st, None, None), (Z, L1.MuonState(over), None, None), (Z, st, over, None),
           (Z, L1.MuonState(over), new, None), (Z, st, None, W.row_ptr[:N]), (Z, st, None, W.col_idx[3:3 + N]),
           (Z, st, None, Z.view(torch.int32).view(-1)[:N]), (Z, st, None, st.m.view(torch.int32).view(-1)[-N:]),
           (Z, st, new, st.m.view(torch.int32).view(-1)[:N]), (Z, st, new, new.view(torch.int32).view(-1)[:N])]
    for O, state, m_out, row_counts in bad:
        with pytest.raises(ValueError):
            L1._muon_writes(W, O, state, m_out, row_counts)
    with pytest.raises(TypeError):
        L1._muon_writes(W, Z.numpy(), st)


@pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")
def test_columns_of_one_buffer_are_no_overlap(lib):
    """Matrices that lie side by side in the rows of one buffer share no element; shifted ones do."""
    at = lambda n: C.c_void_p((1 << 30) + n)  # noqa: E731
    far = C.c_void_p(1 << 44)
    for dtype, e in ((0, 4), (1, 2), (2, 2)):
        wide = dict(dtype=dtype, G=at(0), ldg=24, ldo=24, M=None, M_out=None)
        for o, apart in ((8, True), (16, True), (7, False), (17, False), (1, False), (24 + 8, True), (24 + 4, False),
                         (24 * 7, False), (24 * 8, True)):
            # (not refused: the launch itself fails where there is no GPU)
            assert (muon(lib, O=at(o * e), **wide) != EINVAL) == apart, (dtype, o)
            assert (muon(lib, **{**wide, "G": at(o * e), "O": at(0)}) != EINVAL) == apart, (dtype, o)
            z = dict(dtype=dtype, z=at(0), ld=24, dz=at(o * e), ldd=24, labels=far, old=far, adv=far, stats=C.c_void_p(1 << 45))
            assert (policy(lib, **z) != EINVAL) == apart, (dtype, o)
    side = dict(G=far, ldg=8, O=C.c_void_p(1 << 45), ldo=8, M=at(0), ldm=24)
    assert muon(lib, M_out=at(32), ldmo=24, **side) != EINVAL and muon(lib, M_out=at(28), ldmo=24, **side) == EINVAL
    # a 16-bit gradient of 16 columns' bytes beside the momentum: the same bytes a row
    mixed = dict(dtype=1, O=far, ldo=8, M=at(0), M_out=at(0), ldm=12, ldmo=12, ldg=24)
    assert muon(lib, G=at(32), **mixed) != EINVAL and muon(lib, G=at(30), **mixed) == EINVAL
    assert muon(lib, G=at(34), **mixed) == EINVAL
    # rows of other lengths: refused where the extents meet
    assert muon(lib, G=at(0), ldg=24, O=at(32), ldo=25, M=None, M_out=None) == EINVAL


@pytest.mark.skipif(not NO_GPU, reason="validation calls use placeholder pointers; run without a GPU")
def test_gradient_factors_that_are_refused(lib):
    far = C.c_void_p(1 << 45)
    for s, fine in ((1.0, True), (-65536.0, True), (0.0, True), (nan, False), (inf, False), (-inf, False)):
        # (a sound call is not refused: the launch itself fails where there is no GPU)
        rc = lib.l1csr_policy_loss_scaled(8, 8, 2, P, 8, Q, Q, Q, None, None, 0.2, 0.2, 0.1, s, R, 8, None, far, W, BIG, None)
        assert (rc != EINVAL) == fine, s
        rc = lib.l1csr_preference_loss_scaled(8, 8, 2, P, 8, Q, 2, Q, None, None, 0.1, 0.0, s, R, 8, None, far, W, BIG, None)
        assert (rc != EINVAL) == fine, s
