"""Embedding lookup and its gradients on the GPU against the formulas in 64 bits.

Tolerances.  Forward: one fp32 product (2^-24) and one rounding to the type.  Gradient: a row's n terms are added in fp32 in
some order, at most n - 1 roundings of partial sums that stay below scale * sum |dX|, then a product and a sum with `add`
(2^-24 each) and one rounding to the type.  Where the terms are small whole numbers and the scale a power of two every sum is
exact, and the results have to be equal bit for bit: a term left out or taken twice shows.
"""
import numpy as np
import pytest

import paper_1905_07931_amd as L1

from _helpers import cuda, h

pytestmark = pytest.mark.gpu

HALF_STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}
PAIRS = [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16")]


def _torch():
    import torch
    return torch


def matrix(a, dtype, pad=0, off=0, fill=float("nan")):
    """A [rows][cols] view with a leading dimension of cols + pad, starting `off` elements into its buffer."""
    torch = _torch()
    rows, cols = a.shape
    buf = torch.full((rows * (cols + pad) + off,), fill, dtype=getattr(torch, dtype), device=cuda())
    v = buf[off:].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(getattr(torch, dtype)))
    return v, buf


def h64(x):
    return x.detach().cpu().double().numpy()


def ints(a):
    return _torch().from_numpy(np.asarray(a, np.int32)).to(cuda())


def tokens_of(V, B, rng, kind):
    if kind == "zipf":
        t = np.exp(rng.random(B) * np.log(V + 1)).astype(np.int64) - 1
    elif kind == "one":
        t = np.full(B, V // 2)
    elif kind == "each":
        t = rng.permutation(max(V, B))[:B] % V
    elif kind == "none":
        t = np.full(B, -1)
    else:
        t = rng.integers(0, V, B)
    if kind == "padded":
        t[rng.random(B) < 0.3] = -1
        t[rng.random(B) < 0.1] = V
        t[rng.random(B) < 0.05] = 2 ** 31 - 1
        t[rng.random(B) < 0.05] = -2 ** 31
    return np.clip(t, -2 ** 31, 2 ** 31 - 1)


def lookup(E, t, scale):
    V = E.shape[0]
    X = np.zeros((E.shape[1], t.size))
    good = (t >= 0) & (t < V)
    X[:, good] = scale * E[t[good]].T
    return X


def gradient(dX, t, V, scale):
    """(sum, sum of magnitudes, terms of a row)"""
    dE, size, n = np.zeros((V, dX.shape[0])), np.zeros((V, dX.shape[0])), np.zeros((V, 1))
    for b in np.nonzero((t >= 0) & (t < V))[0]:
        dE[t[b]] += scale * dX[:, b]
        size[t[b]] += abs(scale) * np.abs(dX[:, b])
        n[t[b]] += 1
    return dE, size, n


SHAPES = [(1, 1, 1), (3, 2, 5), (7, 4, 1), (300, 10, 33), (10, 65, 64), (129, 63, 65), (1000, 300, 257), (50, 1001, 130),
          (4097, 8, 1000), (5, 784, 2050), (257, 33, 9001)]


@pytest.mark.parametrize("dtype,out", PAIRS)
@pytest.mark.parametrize("V,D,B", SHAPES)
def test_lookup(V, D, B, dtype, out):
    rng = np.random.default_rng(V + D + B)
    E, _ = matrix(rng.standard_normal((V, D)), dtype, pad=3, off=1)
    t = tokens_of(V, B, rng, "padded" if B > 8 else "any")
    scale = 22.627417
    X, buf = matrix(np.zeros((D, B)), out, pad=5, off=3, fill=7.0)
    got = L1.embedding_fwd(E, ints(t), X=X, scale=scale)
    assert got is X
    want = lookup(h64(E), t, float(np.float32(scale)))
    err = np.abs(h64(X) - want)
    assert (err <= np.abs(want) * (2.0 ** -24 + HALF_STEP[out]) * 1.001 + TINY[out]).all()
    rest = h64(buf[3:].view(D, B + 5)[:, B:])
    assert (rest == 7).all() and (h64(buf[:3]) == 7).all()
    new = L1.embedding_fwd(E, ints(t), scale=scale, dtype=getattr(_torch(), out))
    assert _torch().equal(new, X)


def csr_table(V, D, density, rng, empty=True):
    torch = _torch()
    keep = rng.random((V, D)) < density
    if empty and V > 2:
        keep[1] = False
        keep[2] = True
    dense = np.where(keep, rng.standard_normal((V, D)), 0).astype(np.float32)
    ptr = np.concatenate([[0], keep.sum(1).cumsum()]).astype(np.int32)
    idx = np.nonzero(keep)[1].astype(np.int32)
    W = L1.CSR(V, D, torch.from_numpy(ptr).to(cuda()), torch.from_numpy(np.append(idx, 0).astype(np.int32)).to(cuda()),
               torch.from_numpy(np.append(dense[keep], np.float32(np.nan))).to(cuda()), int(ptr[-1]))
    return W, dense, keep


@pytest.mark.parametrize("density", [0.0, 0.03, 0.5, 1.0])
@pytest.mark.parametrize("V,D,B", [(1, 1, 1), (7, 3, 40), (300, 511, 33), (50, 513, 31), (20, 4100, 65), (129, 1030, 300)])
def test_lookup_in_a_csr_table(V, D, B, density):
    rng = np.random.default_rng(V + D + B)
    W, dense, _ = csr_table(V, D, density, rng)
    t = tokens_of(V, B, rng, "padded" if B > 8 else "any")
    if B > 8 and V > 2:
        t[3], t[4] = 1, 2
    X, buf = matrix(np.ones((D, B)), "float32", pad=3, off=1, fill=7.0)
    L1.embedding_fwd(W, ints(t), X=X, scale=3.0)
    want = lookup(dense.astype(np.float64), t, 3.0)
    assert (np.abs(h64(X) - want) <= np.abs(want) * 2.0 ** -24).all()
    assert (h64(buf[1:].view(D, B + 3)[:, B:]) == 7).all()
    # the same bits as the dense table's
    E, _ = matrix(dense, "float32")
    assert _torch().equal(L1.embedding_fwd(E, ints(t), scale=3.0), X.contiguous())


@pytest.mark.parametrize("kind", ["zipf", "one", "each", "none", "padded"])
@pytest.mark.parametrize("dtype,out", PAIRS)
@pytest.mark.parametrize("V,D,B", [(1, 1, 1), (3, 2, 5), (300, 10, 33), (10, 65, 64), (129, 63, 65), (1000, 300, 257), (5, 100, 2050),
                                   (70, 663, 130), (33, 1290, 70)])
def test_gradient(V, D, B, dtype, out, kind):
    torch = _torch()
    rng = np.random.default_rng(V + D + B)
    t = tokens_of(V, B, rng, kind)
    dX, _ = matrix(rng.standard_normal((D, B)), dtype, pad=3, off=1)
    add, _ = matrix(rng.standard_normal((V, D)) * 3, out, pad=2)
    scale = 1.7
    want, size, n = gradient(h64(dX), t, V, float(np.float32(scale)))

    def check(got, want, base):
        tol = size * (n + 2) * 2.0 ** -24 + (np.abs(base) + np.abs(want)) * 2.0 ** -24
        tol = tol * 1.01 + np.abs(want) * HALF_STEP[out] * 1.001 + TINY[out]
        assert (np.abs(h64(got) - want) <= tol).all()
    dE, buf = matrix(np.full((V, D), np.nan), out, pad=5, off=3, fill=7.0)
    assert L1.embedding_bwd(dX, ints(t), V, dE=dE, scale=scale) is dE
    check(dE, want, 0 * want)
    assert (h64(buf[3:].view(V, D + 5)[:, D:]) == 7).all() and (h64(buf[:3]) == 7).all()
    assert not h64(dE)[n[:, 0] == 0].any()
    got = L1.embedding_bwd(dX, ints(t), V, scale=scale, add=add, dE=torch.empty((V, D), dtype=add.dtype, device=cuda()))
    base = h64(add)
    check(got, want + base, base)
    # in place: the same bits, and rows without tokens untouched
    L1.embedding_bwd(dX, ints(t), V, dE=add, scale=scale, add=add)
    assert torch.equal(add, got)


@pytest.mark.parametrize("kind", ["zipf", "one", "each", "any", "padded"])
@pytest.mark.parametrize("B", [1, 2, 3, 5, 15, 17, 31, 32, 33, 63, 64, 255, 256, 257, 1023, 1024, 1025, 2817, 4096, 8175, 8191, 8192, 8193, 16384, 16385, 24577, 33000])
def test_every_token_is_counted_once(B, kind):
    """Whole numbers: sums are exact, over runs of equal tokens that begin and end anywhere in the groups, and over the
    borders of the ranked runs."""
    torch = _torch()
    rng = np.random.default_rng(B)
    V, D = 97 if kind != "each" else 40000, 6
    t = tokens_of(V, B, rng, kind)
    if kind == "any" and B > 40:
        t[5:B // 2] = 11
    x = rng.integers(-8, 9, (D, B))
    dX = torch.from_numpy(x.astype(np.float32)).to(cuda())
    want = np.zeros((V, D))
    good = (t >= 0) & (t < V)
    np.add.at(want, t[good], 0.5 * x.T[good])
    assert np.array_equal(h64(L1.embedding_bwd(dX, ints(t), V, scale=0.5)), want)
    plan = L1.embedding_plan(ints(t), V)
    # the plan: ranks by (token, position), those of no row last
    words = plan.buf[:4 * 3 * B].view(torch.int32).cpu().numpy()
    key = np.where(good, t, V)
    order = np.lexsort((np.arange(B), key))
    rank = np.empty(B, np.int64)
    rank[order] = np.arange(B)
    assert np.array_equal(words[:B], rank)
    got = L1.embedding_bwd(dX, None, V, scale=0.5, plan=plan)
    assert np.array_equal(h64(got), want)


@pytest.mark.parametrize("density", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("kind", ["zipf", "one", "padded", "none"])
@pytest.mark.parametrize("V,D,B", [(1, 1, 1), (300, 10, 33), (37, 130, 1100), (129, 63, 2050)])
def test_masked_gradient(V, D, B, kind, density):
    torch = _torch()
    rng = np.random.default_rng(V + D + B)
    W, _, keep = csr_table(V, D, density, rng)
    t = tokens_of(V, B, rng, kind)
    dX, _ = matrix(rng.standard_normal((D, B)), "float32", pad=3, off=1)
    nnz = W.nnz
    gv = torch.full((nnz + 2,), 7.0, device=cuda())
    L1.embedding_masked_bwd(W, dX, ints(t), gv=gv, scale=1.7)
    want, size, n = gradient(h64(dX), t, V, float(np.float32(1.7)))
    got = h64(gv)
    tol = (size * (n + 2) * 2.0 ** -24)[keep] * 1.01
    assert (np.abs(got[:nnz] - want[keep]) <= tol).all() and (got[nnz:] == 7).all()
    # the dense gradient's entries, bit for bit
    dense = L1.embedding_bwd(dX, ints(t), V, scale=1.7)
    assert torch.equal(gv[:nnz], dense[torch.from_numpy(keep).to(cuda())])


def test_gradient_against_differences():
    """d/dE of sum(G * X(E)) by central differences of the lookup in exact steps."""
    torch = _torch()
    rng = np.random.default_rng(5)
    V, D, B = 9, 7, 40
    t = tokens_of(V, B, rng, "padded")
    E = rng.integers(-4, 5, (V, D)).astype(np.float32)
    G = torch.from_numpy(rng.integers(-4, 5, (D, B)).astype(np.float32)).to(cuda())
    dE = h64(L1.embedding_bwd(G, ints(t), V, scale=2.0))
    for v in range(V):
        for d in range(0, D, 3):
            f = []
            for step in (1.0, -1.0):
                E2 = E.copy()
                E2[v, d] += step
                X = L1.embedding_fwd(torch.from_numpy(E2).to(cuda()), ints(t), scale=2.0)
                f.append(float((G.double() * X.double()).sum()))
            assert dE[v, d] == (f[0] - f[1]) / 2


@pytest.mark.parametrize("V,B", [(50, 40), (50, 3000), (7, 9000), (2000, 30)])
def test_plan_of_a_larger_table(V, B):
    """The C call with an order that was made for twice the rows: tokens past the table take no part (small whole numbers:
    equal bit for bit), and nothing is written past it."""
    torch, rng = _torch(), np.random.default_rng(7 + V + B)
    t = tokens_of(2 * V, B, rng, "padded")
    X = rng.integers(-8, 9, (20, B)).astype(np.float64)
    dX, _ = matrix(X, "float32")
    plan = L1.embedding_plan(ints(t), 2 * V)
    need = L1.workspace_bytes(L1.OP_EMBEDDING_BWD, V, 20, 0, B)
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device=cuda())
    dE, buf = matrix(np.zeros((V, 20)), "float32", pad=4)
    assert L1.lib().l1csr_embedding_bwd(V, 20, B, 0, dX.data_ptr(), B, plan.buf.data_ptr(), plan.buf.numel(), 2.0, 0, None, 0,
                                        dE.data_ptr(), 24, ws.data_ptr(), need, None) == 0
    torch.cuda.synchronize()
    assert np.array_equal(h64(dE), gradient(X, t, V, 2.0)[0])
    assert bool((ws[need:] == 0x5a).all()) and bool(torch.isnan(buf.view(V, 24)[:, 20:]).all())


def test_special_values_stay_in_their_places():
    torch = _torch()
    V, D, B = 20, 9, 50
    rng = np.random.default_rng(3)
    E = torch.randn(V, D, device=cuda())
    E[3], E[4, 2] = float("nan"), float("inf")
    t = rng.integers(5, V, B)
    t[7] = -1
    assert bool(torch.isfinite(L1.embedding_fwd(E, ints(t))).all())
    t[9], t[10] = 3, 4
    X = L1.embedding_fwd(E, ints(t))
    bad = (~torch.isfinite(X)).cpu().numpy()
    assert bad[:, 9].all() and bad[2, 10] and bad.sum() == D + 1
    dX = torch.randn(D, B, device=cuda())
    dX[:, 7] = float("nan")  # of padding: not used
    dX[1, 9] = float("inf")
    dE = L1.embedding_bwd(dX, ints(t), V)
    bad = (~torch.isfinite(dE)).cpu().numpy()
    assert bad[3, 1] and bad.sum() == 1


@pytest.mark.parametrize("B", [1, 7])
def test_empty_tables_and_batches(B):
    torch = _torch()
    none = torch.empty((0, 5), device=cuda())
    assert not h(L1.embedding_fwd(none, ints([3] * B))).any()
    assert L1.embedding_fwd(torch.ones(4, 5, device=cuda()), ints([])).shape == (5, 0)
    assert L1.embedding_fwd(torch.ones(4, 0, device=cuda()), ints([0] * B)).shape == (0, B)
    assert L1.embedding_bwd(torch.ones(5, B, device=cuda()), ints([0] * B), 0).shape == (0, 5)
    assert L1.embedding_bwd(torch.ones(0, B, device=cuda()), ints([0] * B), 3).shape == (3, 0)
    dE = L1.embedding_bwd(torch.ones(5, 0, device=cuda()), ints([]), 3)
    assert dE.shape == (3, 5) and not h(dE).any()
    add = torch.ones(3, 5, device=cuda())
    assert (h(L1.embedding_bwd(torch.ones(5, 0, device=cuda()), ints([]), 3, add=add)) == 1).all()
    L1.embedding_bwd(torch.ones(5, 0, device=cuda()), ints([]), 3, dE=add, add=add)
    assert (h(add) == 1).all()


def test_rows_past_32_bits():
    """A table of more than 2^31 entries: lookup at its end, and a gradient added in place there."""
    torch = _torch()
    V, D = 40000, 65536
    E = torch.zeros((V, D), dtype=torch.bfloat16, device=cuda())
    E[V - 1] = torch.arange(D, device=cuda()) % 128
    E[V - 2] = 1
    t = ints([V - 1, 0, V - 2, V])
    X = L1.embedding_fwd(E, t)
    assert torch.equal(X[:, 0], E[V - 1]) and torch.equal(X[:, 2], E[V - 2]) and not X[:, 1].any() and not X[:, 3].any()
    dX = torch.ones((D, 4), dtype=torch.bfloat16, device=cuda())
    L1.embedding_bwd(dX, t, V, dE=E, add=E, scale=4.0)
    assert bool((E[V - 1] == (torch.arange(D, device=cuda()) % 128 + 4)).all()) and bool((E[V - 2] == 5).all())
    assert bool((E[0] == 4).all()) and not bool(E[1:V - 2].any())


def test_columns_of_one_buffer():
    torch = _torch()
    buf = torch.zeros(6, 40, device=cuda())
    E, dE = buf[:, :10], buf[:, 20:30]
    E.copy_(torch.randn(6, 10, device=cuda()))
    t = ints([0, 5, 5, 2])
    X = L1.embedding_fwd(E, t)
    L1.embedding_bwd(X, t, 6, dE=dE)
    assert torch.equal(dE[5], 2 * E[5]) and torch.equal(dE[0], E[0]) and not buf[:, 10:20].any() and not buf[:, 30:].any()


def test_refusals():
    torch = _torch()
    dev = cuda()
    E, t = torch.ones(6, 5, device=dev), ints([0, 1, 2])
    X = torch.empty(5, 3, device=dev)
    with pytest.raises(TypeError):
        L1.embedding_fwd(E, t.long())
    with pytest.raises(TypeError):
        L1.embedding_fwd(E.double(), t)
    with pytest.raises(ValueError):
        L1.embedding_fwd(E.t(), t)
    with pytest.raises(ValueError):
        L1.embedding_fwd(E, t, X=torch.empty(5, 4, device=dev))
    with pytest.raises(ValueError):
        L1.embedding_fwd(E, t, X=X.half())
    with pytest.raises(ValueError):
        L1.embedding_fwd(E, t, dtype=torch.float16)
    with pytest.raises(L1.L1CSRError):
        L1.embedding_fwd(E, t, scale=float("nan"))
    with pytest.raises(L1.L1CSRError):  # over the table
        L1.embedding_fwd(E, t, X=E.flatten()[:15].view(5, 3))
    with pytest.raises(ValueError):
        L1.embedding_bwd(X, t, 6, dE=torch.empty(6, 4, device=dev))
    with pytest.raises(ValueError):
        L1.embedding_bwd(X, t, 6, add=torch.empty(5, 5, device=dev))
    with pytest.raises(ValueError):
        L1.embedding_bwd(X, ints([1]), 6)
    with pytest.raises(ValueError):
        L1.embedding_bwd(X, None, 6, plan=L1.embedding_plan(t, 7))
    with pytest.raises(ValueError):
        L1.embedding_bwd(X, None, 6, plan=L1.embedding_plan(ints([1]), 6))
    buf = torch.ones(7, 5, device=dev)
    with pytest.raises(L1.L1CSRError):  # shifted by a row
        L1.embedding_bwd(X, t, 6, dE=buf[1:], add=buf[:6])
    with pytest.raises(L1.L1CSRError):
        L1.embedding_bwd(X, t, 3, dE=X.view(3, 5))
    with pytest.raises((ValueError, TypeError)):
        L1.embedding_fwd(E.cpu(), t)
    with pytest.raises(ValueError):
        L1.embedding_fwd(E, t.cpu())


@pytest.mark.parametrize("B", [70, 9000])
def test_streams_and_reproducibility(B):
    torch = _torch()
    rng = np.random.default_rng(B)
    V, D = 500, 96
    t = ints(tokens_of(V, B, rng, "zipf"))
    dX = torch.randn(D, B, device=cuda())
    want = L1.embedding_bwd(dX, t, V)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = L1.embedding_bwd(dX, t, V, stream=side)
    with torch.cuda.stream(side):
        b = L1.embedding_bwd(dX, t, V)
        plan = L1.embedding_plan(t, V)
    c = L1.embedding_bwd(dX, None, V, plan=plan, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want) and torch.equal(c, want)


def test_graph_replays():
    """Two captured graphs replayed beside each other with eager calls of larger sizes between."""
    torch = _torch()
    rng = np.random.default_rng(1)
    V, D, B = 300, 72, 500
    sets = []
    for seed in range(2):
        t = ints(tokens_of(V, B, rng, "zipf"))
        E = torch.randn(V, D, device=cuda())
        dX = torch.randn(D, B, device=cuda())
        X, dE = torch.empty(D, B, device=cuda()), torch.empty(V, D, device=cuda())
        L1.embedding_fwd(E, t, X=X)
        L1.embedding_bwd(dX, t, V, dE=dE)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L1.embedding_fwd(E, t, X=X, scale=2.0)
            L1.embedding_bwd(dX, t, V, dE=dE, scale=2.0)
        sets.append((g, t, E, dX, X, dE))
    streams = [torch.cuda.Stream() for _ in sets]
    for turn in range(4):
        for g, t, E, dX, X, dE in sets:
            t.copy_(ints(tokens_of(V, B, rng, "padded" if turn % 2 else "zipf")))
            dX.normal_()
            X.fill_(float("nan"))
            dE.fill_(float("nan"))
        torch.cuda.synchronize()
        for s, (g, *_) in zip(streams, sets):
            with torch.cuda.stream(s):
                g.replay()
        L1.embedding_bwd(torch.randn(200, 4000, device=cuda()), ints(rng.integers(0, 50, 4000)), 50)
        torch.cuda.synchronize()
        for g, t, E, dX, X, dE in sets:
            assert torch.equal(X, L1.embedding_fwd(E, t, scale=2.0))
            assert torch.equal(dE, L1.embedding_bwd(dX, t, V, scale=2.0))


def test_graph_keeps_its_plan_when_the_plan_grows():
    """A graph captured with a plan, which is filled again for a larger batch: replays read the order they were captured with."""
    torch, rng = _torch(), np.random.default_rng(11)
    V, D, B = 30, 8, 500
    t = tokens_of(V, B, rng, "zipf")
    X = rng.integers(-8, 9, (D, B)).astype(np.float64)
    dX, _ = matrix(X, "float32")
    plan, dE = L1.embedding_plan(ints(t), V), torch.empty(V, D, device=cuda())
    want = gradient(X, t, V, 1.0)[0]
    L1.embedding_bwd(dX, None, V, dE=dE, plan=plan)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L1.embedding_bwd(dX, None, V, dE=dE, plan=plan)
    larger = tokens_of(V, 9000, rng, "any")
    L1.embedding_plan(ints(larger), V, plan=plan)
    junk = [torch.full((3 * B,), 0x7fffffff, dtype=torch.int32, device=cuda()) for _ in range(64)]
    for _ in range(3):
        dE.fill_(float("nan"))
        graph.replay()
        assert np.array_equal(h64(dE), want)
    big, _ = matrix(rng.integers(-8, 9, (D, 9000)).astype(np.float64), "float32")
    assert np.array_equal(h64(L1.embedding_bwd(big, None, V, plan=plan)), gradient(h64(big), larger, V, 1.0)[0])
    del junk


def test_first_call_of_a_process():
    """The table of element types is filled by the call that needs it, whichever comes first."""
    torch = _torch()
    rng = np.random.default_rng(0)
    W, dense, _ = csr_table(5, 4, 0.5, rng)
    L1._DTYPES.clear()
    X = L1.embedding_fwd(W, ints([1, 2]), X=torch.empty(4, 2, device=cuda()))
    assert np.array_equal(h64(X), dense[[1, 2]].T)


def test_a_plan_that_grows_step_by_step_keeps_little():
    """The buffers that a plan outgrew are together no larger than the one it has."""
    torch, V = _torch(), 50
    t = torch.arange(3000, dtype=torch.int32, device=cuda()) % V
    plan = L1.embedding_plan(t[:1], V)
    for B in range(2, 3001):
        L1.embedding_plan(t[:B], V, plan=plan)
    assert sum(b.numel() for b in plan.outgrown) <= plan.buf.numel() <= 2 * L1.workspace_bytes(L1.OP_EMBEDDING_PLAN, V, 0, 0, 3000)
    dX = torch.ones(4, 3000, device=cuda())
    assert bool((L1.embedding_bwd(dX, None, V, plan=plan) == 60).all())


def test_a_plan_whose_refill_fails_stays_as_it_was():
    torch, V = _torch(), 50
    t = torch.arange(3000, dtype=torch.int32, device=cuda()) % V
    plan = L1.embedding_plan(t[:100], V)
    buf = plan.buf
    for _ in range(2):
        with pytest.raises(L1.L1CSRError):
            L1.embedding_plan(t, (1 << 30) + 1, plan=plan)  # more rows than the order's keys hold
    assert plan.buf is buf and plan.outgrown == [] and (plan.n_rows, plan.B) == (V, 100)
    dX = torch.ones(4, 100, device=cuda())
    assert bool((L1.embedding_bwd(dX, None, V, plan=plan) == 2).all())


@pytest.mark.parametrize("V,D,density", [(1, 700, 0.5), (300, 4097, 0.05), (40, 5000, 1.0), (2000, 1, 0.5), (50, 257, 0.0)])
def test_lookup_of_one_token_in_a_csr_table(V, D, density):
    rng = np.random.default_rng(V + D)
    W, dense, _ = csr_table(V, D, density, rng)
    for t in (0, V - 1, V // 2, V, -1):
        X = L1.embedding_fwd(W, ints([t]), scale=2.0)
        want = 2.0 * dense[t].astype(np.float64) if 0 <= t < V else np.zeros(D)
        assert X.shape == (D, 1) and np.array_equal(h64(X)[:, 0], want)
