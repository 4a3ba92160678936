"""Orthogonalised momentum (muon_update) and the Prox-Muon calls on the GPU against the formulas in 64 bits.

Tolerances are relative to the whole result (2-norm).  Two-part operands hold 22 bits, fp32 ones 24, and both sums are fp32:
the five steps amplify either's roundings alike, so the error of plain fp32 products of the same input measures that
amplification, and 4 times it (two bits) bounds the two-part result's share of it.  To that come the last step's own
roundings, whose size does not depend on what plain products happen to hit: its three terms a x, b x^3, c x^5 are at most
3.4445 + 4.7750 + 2.0315 = 10.3 for x <= 1 against a result of 0.68 or more, 15 times it, and each is off by three roundings
of 2^-23 (two operands and itself): 45 * 2^-23 = 5.4e-6.  (A 1 x 1 matrix, where plain products were 1e-7 off and these
1.3e-6, showed that four roundings of 2^-22 do not cover that.)  One-part products round
their operands by 2^-11 at most, two operands a product and five steps: 5 * 2 * 2^-11 = 4.9e-3 (errors made before the last
steps have flattened the spectrum are those of X, which is kept in two parts).  A 16-bit result rounds by half a step more.
"""
import math

import numpy as np
import pytest

import paper_1905_07931_amd as L1
from paper_1905_07931_amd import synth

from _helpers import bits_equal, cuda, h

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
HALF_STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def _torch():
    import torch
    return torch


def steps_of(U, steps=5, eps=1e-7, dtype=None):
    """The formula, in the matrix's own arithmetic (64 bits by default)."""
    torch = _torch()
    X = U.double()
    tall = X.shape[0] > X.shape[1]
    X = X / (torch.linalg.matrix_norm(X) + eps)
    X = (X.t() if tall else X).contiguous().to(dtype or torch.float64)
    for _ in range(steps):
        G = X @ X.t().contiguous()
        X = A * X + (B * G + C * (G @ G)) @ X
    return (X.t() if tall else X).contiguous()


def rel(x, y):
    n = y.norm()
    return float((x.double() - y).norm() / n) if float(n) else float(x.double().norm())


def bound(U, want, **kw):
    return 4 * rel(steps_of(U, dtype=_torch().float32, **kw), want) + 45 * 2.0 ** -23


def gradient(N, K, seed, spread=True):
    """A few strong directions over noise."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    G = torch.randn((N, K), generator=g, device="cuda") * 0.05
    if spread:
        G += 0.02 * torch.randn((N, 4), generator=g, device="cuda") @ torch.rand((4, K), generator=g, device="cuda")
    return G * 1e-3


# every form: 128 rows or less in one to four row groups, few and many column ranges (summed ahead past 8, looped past
# 192 slices of 64); small, medium and large tiles, cut and whole; steps in groups; one row, one column, odd sizes
SHAPES = [(1, 1), (1, 5), (5, 1), (3, 3), (2, 64), (31, 70), (32, 32), (33, 64), (33, 65), (64, 500), (65, 64), (96, 97),
          (97, 128), (100, 300), (300, 100), (128, 128), (128, 129), (17, 600), (127, 4097), (20, 20000), (9000, 77),
          (129, 200), (129, 129), (200, 9216), (300, 784), (784, 300), (511, 513), (600, 2000), (1777, 1001), (1500, 1500),
          (2100, 2100), (1030, 4100)]


@pytest.mark.parametrize("N,K", SHAPES)
def test_orthogonalize_fp32(N, K):
    G = gradient(N, K, N + 7 * K)
    want = steps_of(G)
    got = L1.orthogonalize(G)
    assert rel(got, want) <= bound(G, want)
    assert bits_equal(h(got), h(L1.orthogonalize(G)))  # reproducible


@pytest.mark.parametrize("N,K", [(4096, 4096), (2048, 9216)])
def test_orthogonalize_large(N, K):
    G = gradient(N, K, 3)
    want = steps_of(G)
    assert rel(L1.orthogonalize(G), want) <= bound(G, want)
    assert rel(L1.orthogonalize(G, precision=L1.F16), want) <= 4.9e-3


@pytest.mark.parametrize("precision", [L1.F32, L1.F16])
@pytest.mark.parametrize("N,K", [(4001, 4090), (4090, 3900), (161, 4100), (161, 4090), (340, 331), (500, 4000), (705, 690), (737, 700),
                                 (2050, 2047)])
def test_orthogonalize_on_either_side_of_the_tile_rules(N, K, precision):
    G = gradient(N, K, 4)
    want = steps_of(G)
    assert rel(L1.orthogonalize(G, precision=precision), want) <= (4.9e-3 if precision == L1.F16 else bound(G, want))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,K", [(1, 1), (1, 5), (33, 65), (100, 300), (129, 200), (784, 300), (600, 2000), (1001, 1777), (1500, 1500),
                                 (2100, 2100)])
def test_orthogonalize_16_bit(N, K, dtype):
    torch = _torch()
    G = (gradient(N, K, N) * 1e3).to(getattr(torch, dtype))
    want = steps_of(G)
    for precision in (None, L1.F32, L1.F16):
        got = L1.orthogonalize(G, precision=precision)
        assert got.dtype == G.dtype
        one = precision == L1.F16 or (precision is None and dtype == "bfloat16")
        # (each element rounds by half a step at most, so the whole does)
        assert rel(got, want) <= (4.9e-3 if one else bound(G, want)) + HALF_STEP[dtype]


@pytest.mark.parametrize("rank", [1, 8])
@pytest.mark.parametrize("N,K", [(33, 65), (128, 300), (300, 784), (1001, 1777)])
def test_rank_deficient(N, K, rank):
    # the directions that G lacks stay empty but for amplified roundings
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(rank)
    G = torch.randn((N, rank), generator=g, device="cuda") @ torch.randn((rank, K), generator=g, device="cuda")
    want = steps_of(G)
    assert rel(L1.orthogonalize(G), want) <= bound(G, want)
    assert rel(L1.orthogonalize(G, precision=L1.F16), want) <= 4.9e-3


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("N,K", [(40, 70), (300, 400), (600, 1500)])
def test_number_of_steps_and_scale(N, K, steps):
    G = gradient(N, K, steps)
    want = 2.5 * steps_of(G, steps=steps)
    assert rel(L1.orthogonalize(G, steps=steps, scale=2.5), want) <= bound(G, want / 2.5, steps=steps)
    assert rel(L1.orthogonalize(G, steps=steps, scale=2.5, precision=L1.F16), want) <= 4.9e-3


def test_diagonal_in_closed_form():
    # a diagonal matrix stays one: every entry goes through the quintic by itself
    torch = _torch()
    d = np.linspace(0.2, 1.0, 150)
    x = d / (np.linalg.norm(d) + 1e-7)
    for _ in range(5):
        x = A * x + B * x ** 3 + C * x ** 5
    G = torch.zeros((150, 200), device="cuda")
    G[torch.arange(150), torch.arange(150)] = torch.from_numpy(d).float().cuda()
    for X in (G, G.t().contiguous(), G[:120, :130].contiguous() * 0 + 0):
        got = L1.orthogonalize(X)
        if not bool(X.any()):
            assert not bool(got.any())
            continue
        diag = h(torch.diagonal(got)).astype(np.float64)
        # 22-bit operands, amplified by a^5 = 485 at most against values of 0.7 or more; nothing off the diagonal
        assert np.abs(diag - x).max() <= 485 * 6 * 2.0 ** -22
        off = got.clone()
        off[torch.arange(150), torch.arange(150)] = 0
        assert not bool(off.any())


@pytest.mark.parametrize("scale", [1e-30, 1e-38, 2.0 ** -140, 1e30, 1e37])
@pytest.mark.parametrize("N,K", [(60, 100), (200, 300)])
def test_magnitudes(N, K, scale):
    torch = _torch()
    G = (gradient(N, K, 1) * 1e3).double() * scale
    G = G.float()
    want = steps_of(G, eps=0.0)
    assert rel(L1.orthogonalize(G, eps=0.0), want) <= bound(G, want, eps=0.0)
    if scale < 1:  # lost against eps: a step of almost nothing, and finite
        assert bool(torch.isfinite(L1.orthogonalize(G, eps=1e-7)).all())


def test_eps_zero_and_non_finite():
    torch = _torch()
    for N, K in ((20, 30), (200, 150)):
        Z = torch.zeros((N, K), device="cuda")
        assert not bool(L1.orthogonalize(Z).any()) and not bool(L1.orthogonalize(Z, eps=0.0).any())
        G = gradient(N, K, 2)
        G[3] = 0  # a row and a column of zeros stay zeros
        G[:, 5] = 0
        got = L1.orthogonalize(G)
        assert not bool(got[3].any()) and not bool(got[:, 5].any())
        half = G * (0.5e-3 / float(G.norm()))
        want = steps_of(half, eps=1e-3)
        assert rel(L1.orthogonalize(half, eps=1e-3), want) <= bound(half, want, eps=1e-3)
        for bad in (float("nan"), float("inf")):
            X = G.clone()
            X[1, 2] = bad
            assert bool(torch.isnan(L1.orthogonalize(X)).all())
            assert bool(torch.isnan(L1.orthogonalize(X, precision=L1.F16)).all())
    assert L1.orthogonalize(torch.empty((0, 5), device="cuda")).shape == (0, 5)
    assert L1.orthogonalize(torch.empty((5, 0), device="cuda")).shape == (5, 0)


def _layer(N, K, density, seed):
    L = synth.fc_layer(N, K, 4, max(1, int(density * N * K)), seed=seed)
    return L1.CSR.from_host(L.row_ptr, L.col_idx, L.vals, K, device=cuda()), L


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("N,K,pad,off", [(1, 1, 0, 0), (33, 65, 3, 1), (300, 100, 1, 2), (130, 300, 5, 3), (700, 650, 2, 1)])
def test_prox_muon_step(N, K, pad, off, nesterov):
    """Strided gradient, momentum and result, carried over three steps."""
    torch = _torch()

    def strided(x, p=pad, o=off):
        buf = torch.full((x.shape[0] * (x.shape[1] + p) + o,), 3.0, device="cuda")
        v = buf[o:].view(x.shape[0], x.shape[1] + p)[:, :x.shape[1]]
        v.copy_(x)
        return buf, v

    W, L = _layer(N, K, 0.2, 11)
    dense = np.zeros((N, K))
    dense[np.repeat(np.arange(N), np.diff(L.row_ptr)), L.col_idx[:L.row_ptr[-1]]] = L.vals[:L.row_ptr[-1]]
    dense = torch.from_numpy(dense).cuda()
    mbuf, m = strided(torch.zeros((N, K), device="cuda"))
    st = L1.MuonState(m, mu=0.9, nesterov=nesterov)
    m64 = torch.zeros((N, K), dtype=torch.float64, device="cuda")
    eta, lam = 0.02, 0.3
    for k in range(3):
        gbuf, G = strided(gradient(N, K, 20 + k), pad + 1, off)
        zbuf, Z = strided(torch.zeros((N, K), device="cuda"), pad + 2, off)
        m_before = m.double().clone()
        back = L1.prox_muon_step(W, G, st, eta, lam, Z=Z)
        assert back is Z
        m64 = 0.9 * m_before + G.double()
        assert bool(((m.double() - m64).abs() <= (m64.abs() + 0.9 * m_before.abs()) * 2.0 ** -23 + 1e-45).all())
        U = (G.double() + 0.9 * m.double()) if nesterov else m.double()
        want = steps_of(U) * math.sqrt(max(1.0, N / K))
        O = L1.orthogonalize(U.float()).double() * math.sqrt(max(1.0, N / K))
        tol = bound(U.float(), steps_of(U.float())) + 2.0 ** -22
        assert rel(O, want) <= tol
        z = dense - eta * want
        Zw = torch.sign(z) * (z.abs() - eta * lam).clamp_min(0)
        # the threshold does not enlarge a difference; Z rounds twice
        assert float((Z.double() - Zw).norm()) <= eta * tol * float(want.norm()) + 2.0 ** -23 * float(z.norm())
        for b, v, p in ((mbuf, m, pad), (gbuf, G, pad + 1), (zbuf, Z, pad + 2)):
            rest = b[off:].view(N, K + p)[:, K:]
            assert bool((rest == 3).all()) and bool((b[:off] == 3).all())
    # m kept, m' elsewhere; Z over the gradient
    kept = m.clone()
    new = torch.empty((N, K), device="cuda")
    G = gradient(N, K, 40)
    a = L1.prox_muon_step(W, G, st, eta, lam, m_out=new)
    assert torch.equal(m, kept)
    b = L1.prox_muon_step(W, G, st, eta, lam, Z=G)
    assert torch.equal(a, b) and torch.equal(m, new)


@pytest.mark.parametrize("N,K", [(40, 90), (300, 200), (700, 700)])
def test_recompress_and_capacity(N, K):
    torch = _torch()
    W, _ = _layer(N, K, 0.3, 5)
    G, m0 = gradient(N, K, 1), gradient(N, K, 2)
    st = L1.MuonState(m0.clone())
    Z = L1.prox_muon_step(W, G, st, 0.05, 0.1)
    want = L1.csr_recompress(Z)
    st2 = L1.MuonState(m0.clone())
    out = L1.prox_muon_recompress(W, G, st2, 0.05, 0.1)
    assert torch.equal(st.m, st2.m)
    n = out.host_nnz()
    assert n == want.host_nnz() and all(bits_equal(x, y) for x, y in zip(out.to_host(), want.to_host()))
    # a capacity that holds the result, and one that does not: the momentum then stays
    st3 = L1.MuonState(m0.clone())
    fit = L1.prox_muon_recompress(W, G, st3, 0.05, 0.1, capacity=n)
    assert torch.equal(st3.m, st.m) and all(bits_equal(x, y) for x, y in zip(fit.to_host(), want.to_host()))
    if n > 1:
        st4 = L1.MuonState(m0.clone())
        with pytest.raises(L1.L1CSRError):
            L1.prox_muon_recompress(W, G, st4, 0.05, 0.1, capacity=n - 1)
        assert torch.equal(st4.m, m0)


@pytest.mark.parametrize("N,K,Bt", [(60, 100, 32), (400, 700, 96)])
def test_fine_tuning_step(N, K, Bt):
    """A policy step of a compressed layer end to end: product, loss and its gradient, weight gradient, Prox-Muon."""
    torch = _torch()
    W, L = _layer(N, K, 0.3, 3)
    X = torch.randn((K, Bt), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    labels = torch.randint(0, N, (Bt,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).to(torch.int32)
    Y = L1.csr_spmm_fwd(W, X)
    old = L1.token_logp(Y, labels) - 0.02
    adv = torch.linspace(-1, 1, Bt, device="cuda")
    stats, dY, _ = L1.policy_loss(Y, labels, old, adv, ref_logp=old, kl_coef=0.1)
    # the gradient of the logits, by the formula
    lp = torch.log_softmax(Y.double(), 0)
    own = lp[labels.long(), torch.arange(Bt, device="cuda")]
    coef = (-adv.double() * (own - old.double()).exp() - 0.1 * torch.expm1(old.double() - own)) / Bt
    want = -lp.exp() * coef
    want[labels.long(), torch.arange(Bt, device="cuda")] += coef
    assert rel(dY, want) <= 1e-5  # (N + 16) 2^-23 of softmax sums
    results = []
    for schedule in ("serial", "two_stream"):
        st = L1.MuonState.zeros((N, K), "cuda")
        out = L1.CSR(N, K, *(torch.empty(s, dtype=t, device="cuda") for s, t in
                             ((N + 1, torch.int32), (N * K, torch.int32), (N * K, torch.float32))))
        bufs = dict(Y=torch.empty_like(Y), dX=torch.empty_like(X), dW=torch.empty((N, K), device="cuda"),
                    csc=L1.CSC.empty(K, W.nnz, "cuda"), out=out)
        L1.l1_step(W, X, dY, 0.02, 0.05, schedule=schedule, adaptive=st, **bufs)
        results.append([bufs["Y"], bufs["dX"], bufs["dW"], st.m] + [torch.from_numpy(a) for a in out.to_host()])
    assert all(torch.equal(a.cpu(), b.cpu()) for a, b in zip(*results))
    G = L1.dense_wgrad(dY, X)
    st = L1.MuonState.zeros((N, K), "cuda")
    ref = L1.prox_muon_recompress(W, G, st, 0.02, 0.05)
    assert torch.equal(results[0][3], st.m.cpu() if results[0][3].device.type == "cpu" else st.m)
    assert all(bits_equal(h(a), b) for a, b in zip(results[0][4:], ref.to_host()))


def test_streams_and_graphs():
    torch = _torch()
    shapes = [(100, 300), (300, 400), (600, 1200)]
    Gs = [gradient(N, K, 1) for N, K in shapes]
    want = [L1.orthogonalize(G) for G in Gs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [L1.orthogonalize(G, stream=side) for G in Gs]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    W, _ = _layer(100, 300, 0.2, 1)
    graphs, outs, ins = [], [], []
    for k in range(2):
        x = [G.clone() for G in Gs]
        m = torch.zeros((100, 300), device="cuda")
        m_out = torch.empty_like(m)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = [L1.orthogonalize(G) for G in x] + [L1.prox_muon_step(W, x[0], L1.MuonState(m), 0.1, 0.1, m_out=m_out)]
        graphs.append(g)
        outs.append(o)
        ins.append((x, m))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        for i, (x, m) in enumerate(ins):
            for G in x:
                G.copy_(torch.randn_like(G) * (1 + i + rep))
            m.copy_(torch.randn_like(m))
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (x, m), o in zip(ins, outs):
            eager = [L1.orthogonalize(G) for G in x]
            eager.append(L1.prox_muon_step(W, x[0], L1.MuonState(m), 0.1, 0.1, m_out=torch.empty_like(m)))
            assert all(torch.equal(a, b) for a, b in zip(o, eager))


@pytest.mark.parametrize("N,K", [(3001, 50), (3001, 200)])
def test_offsets_past_32_bits(N, K):
    """Rows so far apart that offsets pass 2^32 elements: the bits of the same matrix without the gaps."""
    torch = _torch()
    ld = 1500001
    wide = torch.empty((N, ld), dtype=torch.bfloat16, device="cuda")
    G = wide[:, 3:3 + K]
    G.copy_(gradient(N, K, 1))
    want = L1.orthogonalize(G.contiguous())
    assert torch.equal(L1.orthogonalize(G, out=G), want)


@pytest.mark.parametrize("schedule", ["serial", "two_stream"])
def test_captured_step(schedule):
    """l1_step with a MuonState in a graph, replayed with eager steps between: each replay gives the eager result."""
    torch = _torch()
    N, K, Bt = 300, 784, 64
    W, L = _layer(N, K, 0.1, 4)
    gen = torch.Generator(device="cuda").manual_seed(5)
    X, dY = (torch.randn((r, Bt), device="cuda", generator=gen) for r in (K, N))

    def buffers():
        out = L1.CSR(N, K, *(torch.empty(n, dtype=t, device="cuda") for n, t in
                             ((N + 1, torch.int32), (N * K, torch.int32), (N * K, torch.float32))))
        return dict(Y=torch.empty((N, Bt), device="cuda"), dX=torch.empty((K, Bt), device="cuda"),
                    dW=torch.empty((N, K), device="cuda"), csc=L1.CSC.empty(K, W.nnz, "cuda"), out=out)

    a, b = buffers(), buffers()
    sa, sb = L1.MuonState.zeros((N, K), "cuda"), L1.MuonState.zeros((N, K), "cuda")
    run = lambda st, o: L1.l1_step(W, X, dY, 0.02, 0.05, schedule=schedule, adaptive=st, **o)  # noqa: E731
    run(sb, b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(sa, a)
    for rep in range(3):
        X.normal_(generator=gen)
        dY.normal_(generator=gen)
        sa.m.normal_(generator=gen)
        sb.m.copy_(sa.m)
        run(sb, b)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        n = int(b["out"].row_ptr[-1])
        for x, y in zip([sa.m, a["Y"], a["dX"], a["dW"], a["out"].row_ptr, a["out"].col_idx[:n], a["out"].vals[:n]],
                        [sb.m, b["Y"], b["dX"], b["dW"], b["out"].row_ptr, b["out"].col_idx[:n], b["out"].vals[:n]]):
            assert torch.equal(x, y), rep


@pytest.mark.parametrize("N,K", [(0, 5), (5, 0), (0, 0)])
def test_empty_layers(N, K):
    torch = _torch()
    G = torch.empty((N, K), device="cuda")
    assert L1.orthogonalize(G).shape == (N, K)
    W = L1.CSR(N, K, torch.zeros(N + 1, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
               torch.empty(0, device="cuda"), 0)
    st = L1.MuonState.zeros((N, K), "cuda")
    assert L1.prox_muon_step(W, G, st, 0.1, 0.1).shape == (N, K)
    out = L1.prox_muon_recompress(W, G, st, 0.1, 0.1)
    assert out.host_nnz() == 0 and not out.row_ptr.any()


def test_refused_steps_leave_the_momentum():
    torch = _torch()
    W, _ = _layer(20, 30, 0.5, 1)
    G, m0 = gradient(20, 30, 1), gradient(20, 30, 2)
    st = L1.MuonState(m0.clone())
    new = lambda rows=21, n=600: L1.CSR(20, 30, *(torch.empty(k, dtype=t, device="cuda") for k, t in  # noqa: E731
                                                  ((rows, torch.int32), (n, torch.int32), (n, torch.float32))))
    for eta, lam in ((0.0, 0.1), (-0.1, 0.1), (0.1, -0.1), (float("nan"), 0.1), (0.1, float("inf")), (1e39, 0.1), (1e-60, 0.1)):
        for f in (L1.prox_muon_step, L1.prox_muon_recompress):
            with pytest.raises(ValueError):
                f(W, G, st, eta, lam)
    with pytest.raises(ValueError):
        L1.prox_muon_step(W, G, st, 0.1, 0.1, row_counts=torch.empty(19, dtype=torch.int32, device="cuda"))
    inside = new()
    inside.vals = st.m.view(-1)
    twice = new()
    twice.vals = twice.col_idx.view(torch.float32)
    for kw in (dict(out=new(rows=20)), dict(out=new(), capacity=601), dict(out=W), dict(out=inside), dict(out=twice)):
        with pytest.raises(ValueError):
            L1.prox_muon_recompress(W, G, st, 0.1, 0.1, **kw)
    with pytest.raises(L1.L1CSRError):
        L1.prox_muon_recompress(W, G, st, 0.1, 0.1, capacity=-1)
    assert torch.equal(st.m, m0)
    out = L1.prox_muon_recompress(W, G, st, 0.1, 0.1, out=new())
    want = L1.prox_muon_recompress(W, G, L1.MuonState(m0.clone()), 0.1, 0.1)
    assert all(bits_equal(x, y) for x, y in zip(out.to_host(), want.to_host()))


def test_refusals():
    torch = _torch()
    G = gradient(20, 30, 1)
    with pytest.raises(ValueError):
        L1.orthogonalize(G.t())
    with pytest.raises(TypeError):
        L1.orthogonalize(G.double())
    with pytest.raises(ValueError):
        L1.orthogonalize(G, out=torch.empty((20, 31), device="cuda"))
    with pytest.raises(ValueError):
        L1.orthogonalize(G, out=torch.empty((20, 30), device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        L1.orthogonalize(G, precision=L1.BF16X3)
    for kw in (dict(steps=0), dict(steps=L1.MUON_MAX_STEPS + 1), dict(eps=-1.0), dict(scale=float("inf"))):
        with pytest.raises(L1.L1CSRError):
            L1.orthogonalize(G, **kw)
    with pytest.raises(L1.L1CSRError):  # overlapping, not the same matrix
        buf = torch.zeros((21, 30), device="cuda")
        L1.orthogonalize(buf[:20], out=buf[1:])
    with pytest.raises(ValueError):
        L1.orthogonalize(G.cpu())
    W, _ = _layer(20, 30, 0.5, 1)
    with pytest.raises(ValueError):
        L1.prox_muon_step(W, gradient(20, 31, 1), L1.MuonState.zeros((20, 31), "cuda"), 0.1, 0.1)
    with pytest.raises(ValueError):
        L1.prox_muon_step(W, G, L1.MuonState.zeros((20, 29), "cuda"), 0.1, 0.1)
    with pytest.raises(L1.L1CSRError):
        L1.prox_muon_step(W, G, L1.MuonState.zeros((20, 30), "cuda", mu=1.0), 0.1, 0.1)
    with pytest.raises(L1.L1CSRError):  # the momentum is the gradient
        L1.prox_muon_step(W, G, L1.MuonState(G), 0.1, 0.1)


# every form of the products: one workgroup, a step a launch (few ranges, ranges summed ahead), blocks, groups of steps, tiles
FORMS = [(20, 30), (96, 128), (40, 300), (100, 300), (100, 5000), (300, 784), (700, 300), (600, 2000), (1100, 1100)]


@pytest.mark.parametrize("precision", [L1.F32, L1.F16])
@pytest.mark.parametrize("N,K", FORMS)
def test_zero_update_whatever_eps_is(N, K, precision):
    # U = 0 gives X = 0 / (0 + eps): zeros, also where 1 / eps^2 or 1 / eps is past the largest float
    torch = _torch()
    Z = torch.zeros((N, K), device="cuda")
    for eps in (0.0, 2.0 ** -149, 1e-40, 1e-20, 1e-7, 1.0, 3e38):
        assert not bool(L1.orthogonalize(Z, eps=eps, precision=precision).any()), eps


@pytest.mark.parametrize("N,K", [(20, 30), (100, 300), (300, 400)])
def test_zero_update_leaves_the_prox_step_alone(N, K):
    # neither a gradient nor momentum: Z = S(W)
    torch = _torch()
    W, _ = _layer(N, K, 0.3, 2)
    G = torch.zeros((N, K), device="cuda")
    st = L1.MuonState.zeros((N, K), "cuda", eps=1e-20)
    want = L1.prox_l1_step(L1.PROX_DENSE, W, G, 0.02, 0.1)
    assert torch.equal(L1.prox_muon_step(W, G, st, 0.02, 0.1), want) and not bool(st.m.any())
    out = L1.prox_muon_recompress(W, G, st, 0.02, 0.1)
    assert all(bits_equal(x, y) for x, y in zip(out.to_host(), L1.csr_recompress(want).to_host()))


def _full_csr(N, K):
    torch = _torch()
    return L1.CSR(N, K, *(torch.empty(n, dtype=t, device="cuda") for n, t in
                          ((N + 1, torch.int32), (N * K, torch.int32), (N * K, torch.float32))))


def test_recompressing_graphs_side_by_side():
    # two graphs captured on one stream and replayed on two: neither's scratch of the recompression is the other's
    torch = _torch()
    N, K = 300, 784
    W, _ = _layer(N, K, 0.2, 1)
    graphs, ins, outs = [], [], []
    for k in range(2):
        G, m, out = gradient(N, K, k), torch.zeros((N, K), device="cuda"), _full_csr(N, K)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L1.prox_muon_recompress(W, G, L1.MuonState(m), 0.05, 0.3, out=out)
        graphs.append(g)
        ins.append((G, m))
        outs.append(out)
    # eager calls that need more scratch replace what the stream keeps
    W2, _ = _layer(900, 2000, 0.2, 2)
    big = L1.MuonState.zeros((900, 2000), "cuda")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        want = []
        for i, (G, m) in enumerate(ins):
            G.copy_(torch.randn_like(G) * (1 + i + rep))
            m.copy_(torch.randn_like(m))
            st = L1.MuonState(m.clone())
            want.append((L1.prox_muon_recompress(W, G, st, 0.05, 0.3, out=_full_csr(N, K)), st.m))
        L1.prox_muon_recompress(W2, gradient(900, 2000, rep), big, 0.05, 0.3)
        others = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (ref, m), out, (_, m_got) in zip(want, outs, ins):
            n = int(ref.row_ptr[-1])
            assert torch.equal(out.row_ptr, ref.row_ptr) and torch.equal(out.col_idx[:n], ref.col_idx[:n])
            assert torch.equal(out.vals[:n], ref.vals[:n]) and torch.equal(m_got, m)
        assert all(bool((o == 7).all()) for o in others)


@pytest.mark.parametrize("schedule", ["serial", "two_stream"])
def test_captured_steps_side_by_side(schedule):
    torch = _torch()
    N, K, Bt = 300, 784, 64
    W, _ = _layer(N, K, 0.1, 4)
    gen = torch.Generator(device="cuda").manual_seed(6)

    def buffers():
        return dict(Y=torch.empty((N, Bt), device="cuda"), dX=torch.empty((K, Bt), device="cuda"),
                    dW=torch.empty((N, K), device="cuda"), csc=L1.CSC.empty(K, W.nnz, "cuda"), out=_full_csr(N, K))

    def results(st, o):
        n = int(o["out"].row_ptr[-1])
        return [st.m, o["Y"], o["dX"], o["dW"], o["out"].row_ptr, o["out"].col_idx[:n], o["out"].vals[:n]]

    cases = []
    for k in range(2):
        X, dY = (torch.randn((r, Bt), device="cuda", generator=gen) for r in (K, N))
        st, o = L1.MuonState.zeros((N, K), "cuda"), buffers()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L1.l1_step(W, X, dY, 0.02, 0.05, schedule=schedule, adaptive=st, **o)
        cases.append((g, X, dY, st, o))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        want = []
        for g, X, dY, st, o in cases:
            for x in (X, dY, st.m):
                x.normal_(generator=gen)
            ref, ro = L1.MuonState(st.m.clone()), buffers()
            L1.l1_step(W, X, dY, 0.02, 0.05, schedule=schedule, adaptive=ref, **ro)
            want.append(results(ref, ro))
        torch.cuda.synchronize()
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                c[0].replay()
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert all(torch.equal(a, b) for a, b in zip(results(c[3], c[4]), w)), rep


def test_steps_that_would_write_into_the_layer_are_refused():
    torch = _torch()
    N, K = 20, 30
    W, _ = _layer(N, K, 1.0, 1)
    assert W.nnz == N * K
    keep = [x.clone() for x in (W.row_ptr, W.col_idx, W.vals)]
    G, m0 = gradient(N, K, 1), gradient(N, K, 2)
    over = W.vals[:N * K].view(N, K)
    at = lambda x, n: x.view(torch.int32).view(-1)[:n]  # noqa: E731
    st = L1.MuonState(m0.clone())
    Z = torch.empty((N, K), device="cuda")
    for kw in (dict(Z=over), dict(m_out=over), dict(Z=W.col_idx[:N * K].view(torch.float32).view(N, K)),
               dict(row_counts=W.row_ptr[:N]), dict(row_counts=W.col_idx[:N]), dict(Z=Z, row_counts=at(Z, N)),
               dict(row_counts=at(st.m, N))):
        with pytest.raises(ValueError):
            L1.prox_muon_step(W, G, st, 0.1, 0.1, **kw)
    with pytest.raises(ValueError):
        L1.prox_muon_recompress(W, G, st, 0.1, 0.1, O=over)
    for f in (L1.prox_muon_step, L1.prox_muon_recompress):
        with pytest.raises(ValueError):
            f(W, G, L1.MuonState(over), 0.1, 0.1)
    assert torch.equal(st.m, m0) and all(torch.equal(a, b) for a, b in zip(keep, (W.row_ptr, W.col_idx, W.vals)))


@pytest.mark.parametrize("call", ["step", "recompress", "recompress_short"])
def test_calls_without_memory_leave_the_momentum(call, monkeypatch):
    # whichever of a call's allocations fails, the momentum is not stored
    torch = _torch()
    N, K = 300, 200
    W, _ = _layer(N, K, 0.3, 5)
    G, m0 = gradient(N, K, 1), gradient(N, K, 2)
    st = L1.MuonState(m0.clone())
    run = {"step": lambda: L1.prox_muon_step(W, G, st, 0.05, 0.1),
           "recompress": lambda: L1.prox_muon_recompress(W, G, st, 0.05, 0.1),
           "recompress_short": lambda: L1.prox_muon_recompress(W, G, st, 0.05, 0.1, capacity=N * K - 1)}[call]
    empty, left = torch.empty, [0]

    def limited(*a, **kw):
        if left[0] == 0:
            raise torch.OutOfMemoryError("no memory left")
        left[0] -= 1
        return empty(*a, **kw)

    for n in range(20):
        L1._ws_cache.clear()
        left[0] = n
        monkeypatch.setattr(torch, "empty", limited)
        try:
            done = run()
        except torch.OutOfMemoryError:
            done = None
        monkeypatch.setattr(torch, "empty", empty)
        torch.cuda.synchronize()
        if done is not None:
            break
        assert torch.equal(st.m, m0), n
    assert done is not None and n >= 2 and not torch.equal(st.m, m0)


def test_memory_belongs_to_the_calls_stream(monkeypatch):
    # what a call allocates for its work on a stream is allocated in that stream's order
    torch = _torch()
    W, _ = _layer(300, 200, 0.3, 5)
    G, st = gradient(300, 200, 1), L1.MuonState.zeros((300, 200), "cuda")
    torch.cuda.synchronize()
    side, seen, empty = torch.cuda.Stream(), [], torch.empty

    def watched(*a, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **kw)

    monkeypatch.setattr(torch, "empty", watched)
    L1._ws_cache.clear()
    L1.prox_muon_recompress(W, G, st, 0.05, 0.1, stream=side)
    L1.prox_muon_recompress(W, G, st, 0.05, 0.1, capacity=300 * 200 - 1, stream=side)
    L1.prox_muon_step(W, G, st, 0.05, 0.1, stream=side)
    L1.orthogonalize(G, stream=side)
    monkeypatch.setattr(torch, "empty", empty)
    side.synchronize()
    assert len(seen) >= 8 and set(seen) == {side.cuda_stream}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("N,K", [(33, 65), (130, 301), (301, 130)])
def test_columns_of_one_buffer(N, K, dtype):
    # the parts of a fused gradient, their update beside them: the bits of matrices apart, the other columns untouched
    torch = _torch()
    buf = torch.full((N, 4 * K + 3), 7.0, device="cuda", dtype=getattr(torch, dtype))
    G, O = buf[:, K:2 * K], buf[:, 2 * K:3 * K]
    G.copy_(gradient(N, K, 5) * 1e3)
    want = L1.orthogonalize(G.contiguous())
    assert torch.equal(L1.orthogonalize(G, out=O), want) and torch.equal(O, want)
    assert bool((buf[:, :K] == 7).all()) and bool((buf[:, 3 * K:] == 7).all())
    if dtype != "float32":
        return
    W, _ = _layer(N, K, 0.3, 1)
    state = torch.full((N, 3 * K), 5.0, device="cuda")
    m, new, Z = (state[:, i * K:(i + 1) * K] for i in range(3))
    m.copy_(gradient(N, K, 6))
    ref, ref_new = L1.MuonState(m.contiguous()), torch.empty((N, K), device="cuda")
    want = L1.prox_muon_step(W, G, ref, 0.05, 0.1, m_out=ref_new)
    assert torch.equal(L1.prox_muon_step(W, G, L1.MuonState(m), 0.05, 0.1, Z=Z, m_out=new), want)
    assert torch.equal(new, ref_new) and torch.equal(m, ref.m)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("N,K", [(100, 300), (300, 784), (1500, 1500)])
def test_fewer_bits_only_where_asked_for(N, K, dtype):
    torch = _torch()
    G = (gradient(N, K, 8) * 1e3).to(getattr(torch, dtype))
    full = L1.orthogonalize(G, precision=L1.F32)
    assert torch.equal(L1.orthogonalize(G), full) and torch.equal(L1.orthogonalize(G, precision=None), full)
    # the result's rounding is all that a 16-bit matrix loses: half a step an element
    want = steps_of(G)
    assert rel(full, want) <= bound(G, want) + HALF_STEP[dtype]
    assert (min(N, K) <= 128) == torch.equal(L1.orthogonalize(G, precision=L1.F16), full)


def test_step_takes_the_states_precision():
    torch = _torch()
    N, K, Bt = 300, 784, 64
    W, _ = _layer(N, K, 0.1, 4)
    gen = torch.Generator(device="cuda").manual_seed(7)
    X, dY = (torch.randn((r, Bt), device="cuda", generator=gen) for r in (K, N))
    G = L1.dense_wgrad(dY, X)
    updates = {}
    for precision in (L1.F32, L1.F16):
        st, dW = L1.MuonState.zeros((N, K), "cuda", precision=precision), torch.empty((N, K), device="cuda")
        out = _full_csr(N, K)
        L1.l1_step(W, X, dY, 0.02, 0.05, Y=torch.empty((N, Bt), device="cuda"), dX=torch.empty((K, Bt), device="cuda"), dW=dW,
                   csc=L1.CSC.empty(K, W.nnz, "cuda"), out=out, adaptive=st)
        ref, O = L1.MuonState.zeros((N, K), "cuda"), torch.empty((N, K), device="cuda")
        want = L1.prox_muon_recompress(W, G, ref, 0.02, 0.05, O=O, precision=precision)
        assert torch.equal(dW, O) and all(bits_equal(a, b) for a, b in zip(out.to_host(), want.to_host()))
        # a call's own choice goes before the state's
        other = L1.MuonState.zeros((N, K), "cuda", precision=L1.F16)
        assert torch.equal(L1.prox_muon_step(W, G, other, 0.02, 0.05, precision=precision),
                           L1.prox_muon_step(W, G, L1.MuonState.zeros((N, K), "cuda"), 0.02, 0.05, precision=precision))
        updates[precision] = dW
    exact = steps_of(1.95 * G.double())  # mu 0.95 from zero momentum: U = 1.95 G
    assert rel(updates[L1.F32], exact) <= bound(1.95 * G, exact) and rel(updates[L1.F16], exact) <= 4.9e-3
    assert not torch.equal(updates[L1.F32], updates[L1.F16])
    with pytest.raises(ValueError):
        L1.prox_muon_step(W, G, L1.MuonState.zeros((N, K), "cuda", precision=L1.BF16X3), 0.02, 0.05)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("nesterov", [0, 1])
@pytest.mark.parametrize("N,K", FORMS)
def test_momentum_read_but_not_stored(N, K, nesterov, dtype):
    # muon_update with M and without M_out: the update of the call that stores it, and M as it was
    torch = _torch()
    G = (gradient(N, K, 1) * 1e3).to(getattr(torch, dtype))
    code = {"float32": 0, "bfloat16": 1}[dtype]
    M = torch.full((N, K + 3), 9.0, device="cuda")
    M[:, :K] = gradient(N, K, 2) * 1e3
    before = M.clone()
    for precision, op in ((L1.F32, L1.OP_MUON), (L1.F16, L1.OP_MUON_F16)):
        out, new = [torch.empty_like(G) for _ in range(2)], torch.empty((N, K), device="cuda")
        n = L1.workspace_bytes(op, N, K, 0, 0)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        for O, store in zip(out, (None, new)):
            assert L1.lib().muon_update(N, K, code, G.data_ptr(), K, M.data_ptr(), K + 3, None if store is None else store.data_ptr(),
                                        K, 0.9, nesterov, 5, 1e-7, 1.0, precision, O.data_ptr(), K, ws.data_ptr(), n,
                                        torch.cuda.current_stream().cuda_stream) == L1.OK
        assert torch.equal(out[0], out[1]) and torch.equal(M, before)
        m64 = 0.9 * M[:, :K].double() + G.double()
        assert rel(new, m64) <= 2.0 ** -22
        U = (G.double() + 0.9 * new.double()) if nesterov else new.double()
        want = steps_of(U)
        tol = 4.9e-3 if precision == L1.F16 else bound(U.float(), want) + 2.0 ** -22
        assert rel(out[0], want) <= tol + HALF_STEP[dtype]


def _quintic(x):
    return A * x + B * x ** 3 + C * x ** 5


@pytest.mark.parametrize("steps", [8, 9, 12, 16, 20])
@pytest.mark.parametrize("N,K", [(15, 30), (96, 128), (300, 98), (98, 5000), (300, 784), (700, 302), (602, 2000), (1100, 1100)])
def test_many_steps_of_equal_singular_values(N, K, steps):
    """Orthonormal rows (columns): every singular value is s = m^(-1/2) at first and runs through the quintic, and the matrix is
    f^k(s) Q.  An error of the matrix grows by |f'(s)| (in directions that change singular values) or f(s) / s (in those that
    turn vectors) a step, with 18 e^2 of its square (|f''| / 2 <= 18 up to 1.2); a step adds 16 roundings of 2^-23 of its three
    terms (operands as parts, sums, stored parts), the input and its norm 2^-22."""
    torch = _torch()
    m = min(N, K)
    gen = torch.Generator().manual_seed(N + K)
    Q = torch.linalg.qr(torch.randn((max(N, K), m), generator=gen, dtype=torch.float64))[0].cuda()
    Q = (Q if N >= K else Q.t()).contiguous()
    s, e = m ** -0.5, m ** -0.5 * 2.0 ** -22
    for _ in range(steps):
        slope = abs(A + 3 * B * s * s + 5 * C * s ** 4)
        e = max(slope, abs(_quintic(s) / s)) * e + 18 * e * e + 16 * 2.0 ** -23 * (A * s - B * s ** 3 + C * s ** 5)
        s = _quintic(s)
    assert e / s <= 0.02  # (a step more or less is off by far more)
    got = L1.orthogonalize(Q.float() * 3.0, steps=steps, eps=0.0)
    assert rel(got, s * Q) <= e / s


@pytest.mark.parametrize("precision", [L1.F32, L1.F16])
@pytest.mark.parametrize("N,K", [(20, 33), (60, 128), (300, 70), (100, 5000), (200, 784), (250, 900), (600, 2000)])
def test_most_steps(N, K, precision):
    """L1CSR_MUON_MAX_STEPS steps of any matrix.  The quintic maps [0.681, 1.204] (its lowest value past the first maximum, at
    1.050, and that maximum, at 0.554) into itself and lifts smaller values by 3.4 a step, so all singular values end there, a
    step's roundings aside: 16 2^-23 (two parts) or 3 2^-11 (one part) of three terms of 10.3 at most.  The singular vectors stay,
    so G O^T is symmetric: an error that turns vectors grows by (f(s) + f(t)) / (s + t) a step, a product that telescopes to
    1.204 / 0.681 at most, and a step's roundings add 16 2^-23 10.3 / 0.681."""
    torch = _torch()
    G = torch.randn((N, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(N))
    O = L1.orthogonalize(G, steps=L1.MUON_MAX_STEPS, precision=precision).double()
    one = precision == L1.F16 and min(N, K) > 128
    step = (3 * 2.0 ** -11 if one else 16 * 2.0 ** -23) * 10.3
    sv = torch.linalg.svdvals(O.cpu())
    assert 0.681 - step <= float(sv.min()) and float(sv.max()) <= 1.204 + step
    if not one:
        P = (G.double() @ O.t().contiguous()) if N <= K else (O.t().contiguous() @ G.double())
        assert float((P - P.t()).norm() / P.norm()) <= L1.MUON_MAX_STEPS * step / 0.681 * (1.204 / 0.681)
