"""The norms before and after a block with its gate and residual, and their gradients, on the GPU against the formulas in 64
bits.

Tolerances, with E = 2^-24 and every product, sum and rounding counted once.  Forward, with x = alpha a w q y: the factor
alpha a w has 2 roundings and the gate's own (a logistic function: the exponential within 2 E of its value, its sum, the
quotient: 4 E), y q 2 more, their product one: x within 9 E |x|, r' within 9 E |x| + E |r'|.  The sums are double sums of
values within 6 E of theirs, so s is off by the relative size of that error, 6 E |x|_2 / |r'|_2, and its rounding: h within
|s w| 9 E |x| + |h| (4 E + 6 E |x|_2 / |r'|_2).  Backward, u = dh w: t = dr' + s u - (s^2 c) (s r') has terms within 4 E
of theirs and c is a double mean of products within E: t within ET = E (|dr'| + 4 |s u| + 4 |s^2 c s r'| + s^2 C |s r'| + 2 |t|),
C = mean |u r'|.  dy = alpha a w q t - (q^2 e) (q y) likewise, with e a mean of terms within 7 E of their size
M = mean |k y| (|dr'| + |s u| + |s^2 c s r'|), k = alpha a w, and c's error in it.  dgate = alpha t w q y a' has 8 roundings and
the logistic function's 10 E.  The sums over tokens add at most 24 roundings of partial sums (fp32: a thread's vector, a
wave, then double) to the terms' own errors.  One rounding to the type comes on top of each.
"""
import math

import numpy as np
import pytest

import paper_1905_07931_amd as L1

from _helpers import cuda

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -126, "bfloat16": 2.0 ** -126, "float16": 2.0 ** -24}
TYPES = ["float32", "bfloat16", "float16"]


def _torch():
    import torch
    return torch


def h64(x):
    return None if x is None else x.detach().cpu().double().numpy()


def view(a, dtype, pad=0, off=0, fill=float("nan")):
    torch = _torch()
    rows, cols = a.shape
    buf = torch.full((rows * (cols + pad) + off,), fill, dtype=getattr(torch, dtype), device=cuda())
    v = buf[off:].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(getattr(torch, dtype)))
    return v


def vec(a):
    return _torch().from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(cuda())


def act(g, sigmoid):
    if g is None:
        return 1.0, 0.0
    g = g[:, None] if g.ndim == 1 else g
    if not sigmoid:
        return g, np.ones_like(g)
    a = np.where(g >= 0, 1 / (1 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1 + np.exp(-np.abs(g))))
    b = np.where(g >= 0, np.exp(-np.abs(g)) / (1 + np.exp(-np.abs(g))), 1 / (1 + np.exp(-np.abs(g))))
    return a, a * b


def forward(r, y, gate, post, pre, alpha, eps, sigmoid):
    """(r', h, tolerances of both before their rounding)"""
    K = r.shape[0]
    x = np.zeros_like(r)
    if y is not None:
        a, _ = act(gate, sigmoid)
        w = 1.0 if post is None else post[:, None]
        q = 1.0 if post is None else 1 / np.sqrt((y * y).sum(0) / K + eps)
        x = alpha * a * w * (y * q)
    rn = r + x
    tr = 9 * E * np.abs(x) + E * np.abs(rn)
    if pre is None:
        return rn, None, tr, None
    s = 1 / np.sqrt((rn * rn).sum(0) / K + eps)
    hh = rn * s * pre[:, None]
    ratio = np.sqrt((x * x).sum(0)) * s / math.sqrt(K)  # |x|_2 / |r'|_2 where eps is small, less elsewhere
    th = np.abs(s * pre[:, None]) * 9 * E * np.abs(x) + np.abs(hh) * (4 * E + 6 * E * ratio * (1 + ratio))
    return rn, hh, tr, th


def backward(rn, dr, dh, y, gate, post, pre, alpha, eps, sigmoid):
    """{name: (value, tolerance before its rounding)}"""
    K, B = (rn if rn is not None else y).shape
    zero = np.zeros((K, B))
    dr = zero if dr is None else dr
    out = {}
    t, tt = dr, E * np.abs(dr)
    su, fr = zero, zero
    cerr = zero
    if pre is not None:
        u = dh * pre[:, None]
        s = 1 / np.sqrt((rn * rn).sum(0) / K + eps)
        c = (u * rn).sum(0) / K
        C = np.abs(u * rn).sum(0) / K
        su, fr = s * u, s * s * c * (s * rn)
        cerr = E * s * s * C * np.abs(s * rn)
        t = dr + su - fr
        tt = E * (np.abs(dr) + 4 * np.abs(su) + 4 * np.abs(fr) + 2 * np.abs(t)) + cerr
        term = dh * (rn * s)
        out["pre_gain"] = (term.sum(1), 28 * E * np.abs(term).sum(1))
        out["r"] = (t, tt)
    if y is None:
        return out
    a, da = act(gate, sigmoid)
    w = 1.0 if post is None else post[:, None]
    k = alpha * a * w
    q = 1.0 if post is None else 1 / np.sqrt((y * y).sum(0) / K + eps)
    first, second, terr = q * k * t, zero, zero
    if post is not None:
        e = (k * y * t).sum(0) / K
        size = (np.abs(k * y) * (np.abs(dr) + np.abs(su) + np.abs(fr))).sum(0) / K
        second = q * q * e * (q * y)
        terr = q * q * (9 * E * size + (np.abs(k * y) * cerr).sum(0) / K) * np.abs(q * y)
        term = alpha * a * t * (y * q)
        out["post_gain"] = (term.sum(1), (32 * E * np.abs(term) + np.abs(alpha * a * q * y) * tt).sum(1))
    dy = first - second
    out["y"] = (dy, np.abs(q * k) * tt + E * (9 * np.abs(first) + 4 * np.abs(second) + np.abs(dy)) + terr)
    if gate is not None:
        dg = alpha * t * (w * q * y) * da
        tg = np.abs(alpha * (w * q * y) * da) * tt + 18 * E * np.abs(dg)
        out["gate"] = (dg.sum(1), (tg + 24 * E * np.abs(dg)).sum(1)) if gate.ndim == 1 else (dg, tg)
    return out


def close(got, want, tol, dtype, what):
    got = h64(got)
    tol = tol * 1.01 + np.abs(want) * HALF_STEP[dtype] * 1.001 + TINY[dtype]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


def case(K, B, dtype, gate, post, seed, pad=0, off=0):
    rng = np.random.default_rng(seed)
    sizes = np.exp(0.7 * rng.standard_normal((K, 1)))
    s = dict(r=view(rng.standard_normal((K, B)) * sizes, dtype, pad, off), y=view(rng.standard_normal((K, B)) * 0.4, dtype, pad, off),
             dr=view(rng.standard_normal((K, B)), dtype, pad, off), dh=view(rng.standard_normal((K, B)), dtype, pad, off),
             pre=vec(1 + 0.3 * rng.standard_normal(K)), post=vec(0.5 + 0.2 * rng.standard_normal(K)) if post else None, gate=None)
    if gate == "row":
        s["gate"] = vec(0.4 + 0.5 * rng.standard_normal(K))
    elif gate == "full":
        s["gate"] = view(0.4 + rng.standard_normal((K, B)), dtype, pad, off)
    return s


SHAPES = [(1, 1), (2, 3), (10, 1), (10, 4), (64, 7), (100, 8), (300, 65), (784, 33), (1001, 9), (33, 1030), (4097, 2), (257, 257),
          (5, 5000), (9216, 16), (4500, 37), (4500, 13), (5003, 261), (4099, 5), (9000, 3), (2817, 16), (2816, 17), (2049, 15), (2049, 33)]
FORMS = [("none", False, False), ("none", True, False), ("row", True, False), ("row", False, True), ("row", True, True),
         ("full", True, True), ("full", False, False), ("full", True, False)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate,post,sigmoid", FORMS)
@pytest.mark.parametrize("K,B", SHAPES)
def test_forward_and_backward(K, B, gate, post, sigmoid, dtype):
    torch = _torch()
    s = case(K, B, dtype, gate, post, K + B, pad=5, off=3)
    alpha, eps = 0.7, 1e-5
    a32, e32 = float(np.float32(alpha)), float(np.float32(eps))
    kw = dict(gate=s["gate"], post_gain=s["post"], alpha=alpha, eps=eps, sigmoid=sigmoid)
    r64, y64, g64, post64, pre64 = (h64(s[k]) for k in ("r", "y", "gate", "post", "pre"))
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], pre_gain=s["pre"], **kw)
    want_r, want_h, tr, th = forward(r64, y64, g64, post64, pre64, a32, e32, sigmoid)
    close(rn, want_r, tr, dtype, "r'")
    close(hh, want_h, th, dtype, "h")
    r_only, none = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    assert none is None
    close(r_only, want_r, tr, dtype, "r' alone")
    # backward from r' as stored
    rn64 = h64(rn)
    for dr in (s["dr"], None):
        got = L1.residual_norm_bwd(rn, dr, s["dh"], s["y"], pre_gain=s["pre"], **kw)
        want = backward(rn64, h64(dr), h64(s["dh"]), y64, g64, post64, pre64, a32, e32, sigmoid)
        for name in ("r", "y", "gate", "post_gain", "pre_gain"):
            x = getattr(got, name)
            assert (x is None) == (name not in want), name
            if x is not None:
                close(x, *want[name], str(x.dtype).split(".")[1], ("d" + name, dr is None))
    got = L1.residual_norm_bwd(rn, s["dr"], None, s["y"], **kw)
    want = backward(None, h64(s["dr"]), None, y64, g64, post64, None, a32, e32, sigmoid)
    assert got.r is s["dr"] and got.pre_gain is None
    for name in want:
        x = getattr(got, name)
        close(x, *want[name], str(x.dtype).split(".")[1], "d" + name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,B", SHAPES)
def test_the_norm_alone(K, B, dtype):
    s = case(K, B, dtype, "none", False, K, pad=1, off=1)
    eps = float(np.float32(1e-6))
    r, hh = L1.residual_norm_fwd(s["r"], pre_gain=s["pre"])
    assert r is s["r"]
    _, want, _, th = forward(h64(r), None, None, None, h64(s["pre"]), 1.0, eps, False)
    close(hh, want, th, dtype, "h")
    for dr in (None, s["dr"]):
        got = L1.residual_norm_bwd(r, dr, s["dh"], pre_gain=s["pre"])
        assert got.y is None and got.gate is None and got.post_gain is None
        for name, (w, tol) in backward(h64(r), h64(dr), h64(s["dh"]), None, None, None, h64(s["pre"]), 1.0, eps, False).items():
            x = getattr(got, name)
            close(x, w, tol, str(x.dtype).split(".")[1], "d" + name)


@pytest.mark.parametrize("K,B", [(4096, 300), (1000, 2100), (9216, 70), (300, 9000), (20000, 5), (3, 70000), (2500, 1003), (1500, 2101),
                                 (1024, 2500), (1025, 2500), (17000, 1), (40, 66000)])
def test_larger(K, B):
    """Sums over many rows and columns, in several blocks of each."""
    s = case(K, B, "float32", "full", True, 1)
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True)
    eps = float(np.float32(1e-6))
    args = [h64(s[k]) for k in ("y", "gate", "post", "pre")]
    want_r, want_h, tr, th = forward(h64(s["r"]), *args, 1.0, eps, True)
    close(rn, want_r, tr, "float32", "r'")
    close(hh, want_h, th, "float32", "h")
    got = L1.residual_norm_bwd(rn, s["dr"], s["dh"], s["y"], gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True)
    for name, (w, tol) in backward(h64(rn), h64(s["dr"]), h64(s["dh"]), *args, 1.0, eps, True).items():
        close(getattr(got, name), w, tol, "float32", "d" + name)


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e18])
def test_magnitudes(size):
    """Values whose squares leave fp32's range."""
    K, B = 300, 20
    s = case(K, B, "float32", "row", True, 4)
    s["r"] *= size
    s["y"] *= size
    eps = float(np.float32(1e-38))
    args = [h64(s[k]) for k in ("y", "gate", "post", "pre")]
    kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], eps=1e-38)
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    want_r, want_h, tr, th = forward(h64(s["r"]), *args, 1.0, eps, False)
    close(rn, want_r, tr, "float32", "r'")
    close(hh, want_h, th, "float32", "h")
    got = L1.residual_norm_bwd(rn, s["dr"], s["dh"], s["y"], **kw)
    for name, (w, tol) in backward(h64(rn), h64(s["dr"]), h64(s["dh"]), *args, 1.0, eps, False).items():
        close(getattr(got, name), w, tol, "float32", "d" + name)


def test_a_block_that_takes_back_the_residual():
    """r' is a thousandth of r and of x: the sum over r'^2 from its three parts keeps its digits."""
    rng = np.random.default_rng(0)
    K, B = 1000, 30
    y = rng.standard_normal((K, B))
    q = 1 / np.sqrt((y * y).mean(0))
    s = dict(y=view(y, "float32"), post=vec(np.ones(K)), pre=vec(np.ones(K)))
    s["r"] = view(-y * q + 1e-3 * rng.standard_normal((K, B)), "float32")
    eps = float(np.float32(1e-12))
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], post_gain=s["post"], pre_gain=s["pre"], eps=1e-12)
    want_r, want_h, tr, th = forward(h64(s["r"]), h64(s["y"]), None, h64(s["post"]), h64(s["pre"]), 1.0, eps, False)
    close(rn, want_r, tr, "float32", "r'")
    close(hh, want_h, th, "float32", "h")


@pytest.mark.parametrize("dtype", TYPES)
def test_zero_columns_and_special_values(dtype):
    torch = _torch()
    s = case(100, 21, dtype, "full", True, 6)
    s["r"][:, 3], s["y"][:, 3], s["dh"][:, 3], s["dr"][:, 3] = 0, 0, 0, 0  # padding
    kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True)
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    got = L1.residual_norm_bwd(rn, s["dr"], s["dh"], s["y"], **kw)
    for x in (rn, hh, got.r, got.y, got.gate):
        assert bool(torch.isfinite(x).all()) and not bool(x[:, 3].any())
    s["r"][7, 5], s["y"][9, 6] = float("nan"), float("inf")
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    good = [b for b in range(21) if b not in (5, 6)]
    assert bool(torch.isfinite(hh[:, good]).all()) and bool(torch.isnan(hh[:, 5]).all()) and bool(torch.isnan(hh[9, 6]))
    assert int(torch.isnan(rn[:, 5]).sum()) == 1
    # large gates: the logistic function at its ends
    s = case(50, 9, dtype, "full", False, 7)
    s["gate"][:, 0], s["gate"][:, 1], s["gate"][:, 2], s["gate"][:, 3] = 1000.0, -1000.0, float("inf"), -float("inf")
    rn, _ = L1.residual_norm_fwd(s["r"], s["y"], gate=s["gate"], sigmoid=True)
    d = L1.residual_norm_bwd(rn, s["dr"], None, s["y"], gate=s["gate"], sigmoid=True)
    whole = (s["r"].float() + s["y"].float()).to(s["r"].dtype)
    for c in (0, 2):
        assert torch.equal(rn[:, c], whole[:, c]) and torch.equal(d.y[:, c], s["dr"][:, c])
    for c in (1, 3):
        assert torch.equal(rn[:, c], s["r"][:, c]) and not bool(d.y[:, c].any())
    assert not bool(d.gate[:, :4].any())


def test_gradients_against_differences():
    """Central differences of the forward pass in fp32 (loss: a fixed linear function of r' and h)."""
    torch = _torch()
    K, B = 12, 6
    s = case(K, B, "float32", "full", True, 11)
    R, H = torch.randn(K, B, device=cuda()).double(), torch.randn(K, B, device=cuda()).double()

    def loss(**change):
        a = dict(s, **change)
        rn, hh = L1.residual_norm_fwd(a["r"], a["y"], gate=a["gate"], post_gain=a["post"], pre_gain=a["pre"], alpha=0.8, sigmoid=True)
        return float((rn.double() * R).sum() + (hh.double() * H).sum()), rn
    _, rn = loss()
    d = L1.residual_norm_bwd(rn, R.float(), H.float(), s["y"], gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], alpha=0.8,
                             sigmoid=True)
    step = 2.0 ** -7
    for name, grad in (("r", d.r), ("y", d.y), ("gate", d.gate), ("post", d.post_gain), ("pre", d.pre_gain)):
        flat = grad.contiguous().flatten()
        for i in range(0, flat.numel(), 5):
            two = []
            for sign in (1, -1):
                x = s[name].contiguous().clone().flatten()
                x[i] += sign * step
                two.append(loss(**{name: x.view_as(grad)})[0])
            # third derivatives times step^2 / 6 (of order 10 here), and the outputs' 2^-24 (values up to 4, 144 of them) over the step
            assert abs((two[0] - two[1]) / (2 * step) - float(flat[i])) < 10 * step ** 2 + 144 * 4 * E / step, (name, i)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,B", [(1, 9), (100, 3), (300, 70), (1000, 700), (5000, 37), (4500, 261)])
def test_in_place(K, B, dtype):
    torch = _torch()
    s = case(K, B, dtype, "full", True, 9, pad=3)
    kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True)
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    for ro, ho in (("r", "y"), ("y", "r"), ("r", None), (None, "y")):
        t = {k: s[k].clone() for k in ("r", "y")}
        a, b = L1.residual_norm_fwd(t["r"], t["y"], r_out=t.get(ro), h=t.get(ho), **kw)
        assert torch.equal(a, rn) and torch.equal(b, hh)
    r2 = s["r"].clone()
    _, h1 = L1.residual_norm_fwd(s["r"], pre_gain=s["pre"])
    assert torch.equal(L1.residual_norm_fwd(r2, pre_gain=s["pre"], h=r2)[1], h1)
    want = L1.residual_norm_bwd(rn, s["dr"], s["dh"], s["y"], **kw)
    for into in ("dr", "dh"):
        t = {k: s[k].clone() for k in ("dr", "dh", "y", "gate")}
        got = L1.residual_norm_bwd(rn, t["dr"], t["dh"], t["y"], dr=t[into], dy=t["y"], dgate=t["gate"], **dict(kw, gate=t["gate"]))
        for name in ("r", "y", "gate", "post_gain", "pre_gain"):
            assert torch.equal(getattr(got, name), getattr(want, name)), name


def test_padding_is_left_alone():
    torch = _torch()
    K, B, pad = 37, 21, 6
    s = case(K, B, "bfloat16", "full", True, 2)
    bufs = [torch.full((K, B + pad), 7.0, dtype=torch.bfloat16, device=cuda()) for _ in range(5)]
    v = [b[:, :B] for b in bufs]
    kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"])
    L1.residual_norm_fwd(s["r"], s["y"], r_out=v[0], h=v[1], **kw)
    L1.residual_norm_bwd(v[0], s["dr"], s["dh"], s["y"], dr=v[2], dy=v[3], dgate=v[4], **kw)
    assert all(bool((b[:, B:] == 7).all()) for b in bufs)


@pytest.mark.parametrize("K,B", [(0, 5), (5, 0), (0, 0)])
def test_nothing_to_do(K, B):
    torch = _torch()
    z = lambda: torch.zeros(K, B, device=cuda())  # noqa: E731
    g = torch.ones(K, device=cuda())
    rn, hh = L1.residual_norm_fwd(z(), z(), gate=g, post_gain=g, pre_gain=g)
    assert rn.shape == hh.shape == (K, B)
    d = L1.residual_norm_bwd(rn, z(), z(), z(), gate=g, post_gain=g, pre_gain=g)
    for x in (d.gate, d.post_gain, d.pre_gain):
        assert x.shape == (K,) and not bool(x.any())


def test_refusals():
    torch = _torch()
    r, y, g = torch.ones(6, 5, device=cuda()), torch.ones(6, 5, device=cuda()), torch.ones(6, device=cuda())
    F, Bk = L1.residual_norm_fwd, L1.residual_norm_bwd
    for call in (lambda: F(r), lambda: F(r, post_gain=g, pre_gain=g), lambda: F(r, gate=g, pre_gain=g), lambda: F(r, y[:5]),
                 lambda: F(r, y.half()), lambda: F(r, y, post_gain=g[:5]), lambda: F(r, y, gate=torch.ones(5, device=cuda())),
                 lambda: F(r, y, h=y.clone()), lambda: F(r, pre_gain=g, r_out=y), lambda: F(r, y, gate=y.half()),
                 lambda: Bk(r, None, None, y), lambda: Bk(r, r, r), lambda: Bk(r, None, y, pre_gain=None), lambda: Bk(r, y, pre_gain=g),
                 lambda: Bk(r, y, None, y, dr=r), lambda: Bk(r, None, y, pre_gain=g, dy=r), lambda: F(r.t()[:, :3], pre_gain=g)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        F(r, y, post_gain=g.double())
    z = torch.ones(6, 5, device=cuda())
    for call in (lambda: F(r, y, eps=0.0, post_gain=g), lambda: F(r, y, eps=math.nan, post_gain=g), lambda: F(r, y, alpha=math.inf),
                 lambda: F(r, y, pre_gain=g, r_out=z, h=z), lambda: F(r, y, gate=z, r_out=z), lambda: F(r, y, r_out=r, pre_gain=r.view(-1)[:6]),
                 lambda: Bk(r, z, y, pre_gain=g, dr=r), lambda: Bk(r, z, None, y, dy=z)):
        with pytest.raises(L1.L1CSRError):
            call()


def test_streams_graphs_and_reproducibility():
    torch = _torch()
    sets = []
    for K, B in ((300, 70), (1000, 1100)):
        s = case(K, B, "float32", "full", True, K)
        o = [torch.empty(K, B, device=cuda()) for _ in range(5)]

        def step(s=s, o=o, stream=None):
            kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True, stream=stream)
            L1.residual_norm_fwd(s["r"], s["y"], r_out=o[0], h=o[1], **kw)
            d = L1.residual_norm_bwd(o[0], s["dr"], s["dh"], s["y"], dr=o[2], dy=o[3], dgate=o[4], **kw)
            return [*o, d.post_gain, d.pre_gain]
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = step()
        sets.append((g, s, res, step))
    streams = [torch.cuda.Stream() for _ in sets]
    for turn in range(4):
        for _, s, res, _ in sets:
            s["r"].normal_()
            s["dh"].normal_()
            for x in res:
                x.fill_(float("nan"))
        torch.cuda.synchronize()
        for st, (g, *_) in zip(streams, sets):
            with torch.cuda.stream(st):
                g.replay()
        big = torch.randn(2000, 3000, device=cuda())
        L1.residual_norm_fwd(big, big, pre_gain=torch.ones(2000, device=cuda()), post_gain=torch.ones(2000, device=cuda()))
        torch.cuda.synchronize()
        kept = [[x.clone() for x in res] for _, _, res, _ in sets]
        for (_, _, _, step), k in zip(sets, kept):
            eager = step(stream=streams[1])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, k))


# shapes that take the strips and shapes that take the two passes, of vectors and of single columns
BOTH_WAYS = [(50, 9), (300, 2), (5003, 9), (9000, 3)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("K,B", BOTH_WAYS)
def test_logistic_gates_at_the_ends_of_their_type(K, B, post, dtype):
    """A gate of the type's lowest value is closed, one of its highest open, and neither touches anything else."""
    torch = _torch()
    for kind in ("full", "row"):
        s = case(K, B, dtype, kind, post, 7)
        top = torch.finfo(s["gate"].dtype).max
        at = (slice(None), (0, 1)) if kind == "full" else ((3, K - 1),)  # open, closed: tokens, or features
        s["gate"][at] = torch.tensor([top, -top], dtype=s["gate"].dtype, device=cuda())
        kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True)
        rn, hh = L1.residual_norm_fwd(s["r"], s["y"], **kw)
        d = L1.residual_norm_bwd(rn, s["dr"], s["dh"], s["y"], **kw)
        for x in (rn, hh, d.r, d.y, d.gate, d.pre_gain, *([d.post_gain] if post else [])):
            assert bool(torch.isfinite(x).all()), kind
        assert not bool(d.gate[at].any())
        opened, closed = ((slice(None), 0), (slice(None), 1)) if kind == "full" else (3, K - 1)
        assert torch.equal(rn[closed], s["r"][closed])
        if not post:  # (with a post gain y's part in its own mean has a gradient too)
            assert torch.equal(rn[opened], (s["r"].float() + s["y"].float()).to(s["r"].dtype)[opened])
            assert torch.equal(d.y[opened], d.r[opened]) and not bool(d.y[closed].any())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [1e-12, 1e12, 1e20, 1e30])
@pytest.mark.parametrize("K,B", [(300, 20), (2000, 24), (10, 1), (5003, 21), (9000, 3)])
def test_magnitudes_in_strips_and_passes(K, B, size, dtype):
    """Values whose squares leave fp32's range, in the types that have them."""
    s = case(K, B, dtype, "row", True, 4)
    s["r"] *= size
    s["y"] *= size
    eps = float(np.float32(1e-38))
    args = [h64(s[k]) for k in ("y", "gate", "post", "pre")]
    kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], eps=1e-38)
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    want_r, want_h, tr, th = forward(h64(s["r"]), *args, 1.0, eps, False)
    close(rn, want_r, tr, dtype, "r'")
    close(hh, want_h, th, dtype, "h")
    got = L1.residual_norm_bwd(rn, s["dr"], s["dh"], s["y"], **kw)
    for name, (w, tol) in backward(h64(rn), h64(s["dr"]), h64(s["dh"]), *args, 1.0, eps, False).items():
        x = getattr(got, name)
        close(x, w, tol, str(x.dtype).split(".")[1], "d" + name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,B", [(300, 20), (2000, 24), (10, 1), (5003, 21), (9000, 3)])
def test_a_block_whose_gain_takes_it_past_the_squares(K, B, dtype):
    """h comes from the unrounded r', whose squares leave fp32 (and which leaves fp16 itself)."""
    s = case(K, B, dtype, "none", True, 5)
    s["post"] *= 1e25
    eps = float(np.float32(1e-6))
    _, hh = L1.residual_norm_fwd(s["r"], s["y"], post_gain=s["post"], pre_gain=s["pre"])
    _, want, _, th = forward(h64(s["r"]), h64(s["y"]), None, h64(s["post"]), h64(s["pre"]), 1.0, eps, False)
    close(hh, want, th, dtype, "h")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,B", [(300, 20), (5003, 21)])
def test_infinite_residuals_and_gates(K, B, dtype):
    """r' is infinite where one of its terms is: its column's h is 0 but there, whatever the other term; where r' is NaN (both
    infinite, of unlike signs) the column is."""
    torch = _torch()
    inf = float("inf")
    s = case(K, B, dtype, "full", True, 8)
    #          column: r, gate, y at row 7
    put = {3: (inf, 1, -1), 4: (-inf, 1, 1), 5: (inf, 1, 0), 6: (inf, 0, 1), 8: (0, inf, 1), 9: (2, inf, -1), 10: (inf, inf, 1)}
    for c, (r, gate, y) in put.items():
        s["r"][7, c], s["gate"][7, c], s["y"][7, c] = r, gate, y
    s["r"][7, 12], s["gate"][7, 12], s["y"][7, 12] = -inf, inf, 1
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], gate=s["gate"], post_gain=s["post"].abs_(), pre_gain=s["pre"])
    others = [k for k in range(K) if k != 7]
    for c, (r, gate, y) in put.items():
        assert float(rn[7, c]) == (r if abs(r) == inf else y * gate), c
        assert bool(torch.isnan(hh[7, c])) and not bool(hh[others, c].any()), c
    assert bool(torch.isnan(rn[7, 12])) and bool(torch.isnan(hh[:, 12]).all())
    rest = [c for c in range(B) if c not in put and c != 12]
    assert bool(torch.isfinite(hh[:, rest]).all()) and bool(torch.isfinite(rn[others]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["none", "row", "full"])
@pytest.mark.parametrize("K,B", [(300, 20), (50, 2), (5003, 21), (9000, 3)])
def test_a_block_without_a_norm_has_a_gradient_without_its_values(K, B, kind, dtype):
    """dy = alpha a t: an infinity or a NaN in y does not reach it."""
    torch = _torch()
    s = case(K, B, dtype, kind, False, 13)
    kw = dict(gate=s["gate"], alpha=0.5)
    y = s["y"].clone()
    y[4, 1], y[6, 0], y[K - 1, B - 1] = float("inf"), float("nan"), -float("inf")
    for more in (dict(dh=s["dh"], pre_gain=s["pre"]), {}):
        want = L1.residual_norm_bwd(s["r"], s["dr"], y=s["y"], **more, **kw)
        got = L1.residual_norm_bwd(s["r"], s["dr"], y=y, **more, **kw)
        assert torch.equal(got.y, want.y) and torch.equal(got.r, want.r)


# The tests above with small shapes run in strips; these are the same in two passes (the only way with a workspace forward).

@pytest.mark.parametrize("K,B", [(5003, 30), (4500, 261), (9000, 3)])
def test_passes_of_a_block_that_takes_back_the_residual(K, B):
    """r' is a thousandth of r and of x: the sum over r'^2 from its three parts keeps its digits.  The gain is 1, so x = y there
    without a rounding; a part has at most K + 8 roundings of 2^-53 (its products, sums and the joining) and all are at most R^2 |r'|^2, R^2 =
    (|r| + |x|)^2 / |r'|^2 (4e6): s is within (K + 8) 2^-54 R^2 of its own (q's own error moves r, x and r' together: R, not
    R^2, times as little), and h's entries have those of r' besides."""
    rng = np.random.default_rng(0)
    y = rng.standard_normal((K, B))
    q = 1 / np.sqrt((y * y).mean(0))
    s = dict(y=view(y, "float32"), post=vec(np.ones(K)), pre=vec(np.ones(K)))
    s["r"] = view(-y * q + 1e-3 * rng.standard_normal((K, B)), "float32")
    eps = float(np.float32(1e-12))
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], post_gain=s["post"], pre_gain=s["pre"], eps=1e-12)
    r64, y64 = h64(s["r"]), h64(s["y"])
    want_r, want_h, tr, _ = forward(r64, y64, None, h64(s["post"]), h64(s["pre"]), 1.0, eps, False)
    close(rn, want_r, tr, "float32", "r'")
    x, size = np.abs(want_r - r64), np.sqrt((want_r ** 2).sum(0))
    R2 = (np.sqrt((r64 ** 2).sum(0)) + np.sqrt((x ** 2).sum(0))) ** 2 / size ** 2
    scale = np.sqrt(K) / size  # s without eps, no smaller
    close(hh, want_h, scale * tr + np.abs(want_h) * (4 * E + (K + 8) * 2.0 ** -54 * R2), "float32", "h")


@pytest.mark.parametrize("dtype", TYPES)
def test_passes_of_zero_columns_and_special_values(dtype):
    torch = _torch()
    s = case(5003, 21, dtype, "full", True, 6)
    s["r"][:, 3], s["y"][:, 3], s["dh"][:, 3], s["dr"][:, 3] = 0, 0, 0, 0  # padding
    kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True)
    rn, hh = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    got = L1.residual_norm_bwd(rn, s["dr"], s["dh"], s["y"], **kw)
    for x in (rn, hh, got.r, got.y, got.gate):
        assert bool(torch.isfinite(x).all()) and not bool(x[:, 3].any())
    s["r"][7, 5], s["y"][9, 6], s["y"][5000, 20] = float("nan"), float("inf"), float("nan")
    bad = (5, 6, 20)
    good = [b for b in range(21) if b not in bad]
    rn2, hh2 = L1.residual_norm_fwd(s["r"], s["y"], **kw)
    got2 = L1.residual_norm_bwd(rn2, s["dr"], s["dh"], s["y"], **kw)
    for a, b in ((rn2, rn), (hh2, hh), (got2.r, got.r), (got2.y, got.y), (got2.gate, got.gate)):
        assert torch.equal(a[:, good], b[:, good])  # the other columns have the same bits
    for c in bad:
        assert bool(torch.isnan(hh2[:, c]).all())
    assert int(torch.isnan(rn2[:, 5]).sum()) == 1
    # large gates: the logistic function at its ends
    s = case(4500, 9, dtype, "full", False, 7)
    s["gate"][:, 0], s["gate"][:, 1], s["gate"][:, 2], s["gate"][:, 3] = 1000.0, -1000.0, float("inf"), -float("inf")
    rn, _ = L1.residual_norm_fwd(s["r"], s["y"], gate=s["gate"], sigmoid=True)
    d = L1.residual_norm_bwd(rn, s["dr"], None, s["y"], gate=s["gate"], sigmoid=True)
    whole = (s["r"].float() + s["y"].float()).to(s["r"].dtype)
    for c in (0, 2):
        assert torch.equal(rn[:, c], whole[:, c]) and torch.equal(d.y[:, c], s["dr"][:, c])
    for c in (1, 3):
        assert torch.equal(rn[:, c], s["r"][:, c]) and not bool(d.y[:, c].any())
    assert not bool(d.gate[:, :4].any())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_passes_in_graphs_beside_each_other(dtype):
    """Forward and backward captured twice and replayed on two streams, with an eager call of two passes between."""
    torch = _torch()
    sets = []
    for K, B in ((5003, 70), (4500, 261)):
        s = case(K, B, dtype, "full", True, K)
        o = [torch.empty(K, B, dtype=s["r"].dtype, device=cuda()) for _ in range(5)]

        def step(s=s, o=o, stream=None):
            kw = dict(gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], sigmoid=True, stream=stream)
            L1.residual_norm_fwd(s["r"], s["y"], r_out=o[0], h=o[1], **kw)
            d = L1.residual_norm_bwd(o[0], s["dr"], s["dh"], s["y"], dr=o[2], dy=o[3], dgate=o[4], **kw)
            return [*o, d.post_gain, d.pre_gain]
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = step()
        sets.append((g, s, res, step))
    streams = [torch.cuda.Stream() for _ in sets]
    big, gain = torch.randn(6000, 300, device=cuda()).to(sets[0][1]["r"].dtype), torch.ones(6000, device=cuda())
    for turn in range(4):
        for _, s, res, _ in sets:
            s["r"].normal_()
            s["dh"].normal_()
            for x in res:
                x.fill_(float("nan"))
        torch.cuda.synchronize()
        for st, (g, *_) in zip(streams, sets):
            with torch.cuda.stream(st):
                g.replay()
        rn, _ = L1.residual_norm_fwd(big, big, post_gain=gain, pre_gain=gain)
        L1.residual_norm_bwd(rn, big, big, big, post_gain=gain, pre_gain=gain)
        torch.cuda.synchronize()
        kept = [[x.clone() for x in res] for _, _, res, _ in sets]
        for (_, _, _, step), k in zip(sets, kept):
            eager = step(stream=streams[1])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, k))
