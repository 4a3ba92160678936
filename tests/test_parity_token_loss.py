"""Token log-probabilities, the clipped policy loss and the preference loss on the GPU against the formulas in 64 bits.

Tolerances.  A column's sum of exponentials has C positive terms, each within (|t| + 4) 2^-24 of its value (one rounding of
the exponent t = (z - max) log2 e, one of the exponential, one of a rescaling), and is added in some order with at most
C - 1 roundings and as many rescalings: its relative error is below (2 C + 16) 2^-24 =: ES, the terms with a large |t| being
too small to count.  lp adds roundings of itself and of the logarithm: |lp error| <= ES + 2^-22 (1 + |lp|) =: EL.  A
probability is within ES + (|log p| + 4) 2^-22 =: EP of its value, a coefficient within 4 (EL + 2^-22) of its scale (the
ratio's or the reference's exponential, a few products), and dz rounds once to its type.
"""
import math

import numpy as np
import pytest

import paper_1905_07931_amd as L1

from _helpers import cuda, h

pytestmark = pytest.mark.gpu

HALF_STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -126, "bfloat16": 2.0 ** -126, "float16": 2.0 ** -24}  # a result below rounds by an absolute step
TYPES = ["float32", "bfloat16", "float16"]


def _torch():
    import torch
    return torch


def es(C):
    return (2 * C + 16) * 2.0 ** -24


def el(C, lp):
    return es(C) + 2.0 ** -22 * (1 + np.abs(lp))


def logits(C, B, dtype, seed, pad=0, off=0):
    """A [C][B] view with a leading dimension of B + pad, starting `off` elements into its buffer."""
    torch = _torch()
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((C, B)) * 2
    labels = rng.integers(0, C, B)
    z[labels, np.arange(B)] += rng.uniform(0, 2 + math.log(C), B)
    buf = torch.full((C * (B + pad) + off,), float("nan"), dtype=getattr(torch, dtype), device=cuda())
    v = buf[off:].view(C, B + pad)[:, :B]
    v.copy_(torch.from_numpy(z).to(getattr(torch, dtype)))
    return v, torch.from_numpy(labels.astype(np.int32)).to(cuda()), v.cpu().double().numpy(), labels


def vec(a):
    return _torch().from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(cuda())


def ref_logp(z, labels, counts):
    """(lp, softmax) in 64 bits; the columns that do not count are 0."""
    lp, p = np.zeros(z.shape[1]), np.zeros(z.shape)
    for b in np.nonzero(counts)[0]:
        m = z[:, b].max()
        e = np.exp(z[:, b] - m)
        lp[b] = z[labels[b], b] - m - math.log(e.sum())
        p[:, b] = e / e.sum()
    return lp, p


def ref_policy(lp, counts, w, old, adv, ref, lo, hi, beta):
    w = np.where(counts, w, 0.0)
    sw = w.sum()
    pg, kl, off, d = (np.zeros_like(lp) for _ in range(4))
    for b in np.nonzero(counts)[0]:
        r = math.exp(lp[b] - old[b])
        off[b] = (adv[b] > 0 and r > 1 + hi) or (adv[b] < 0 and r < 1 - lo)
        pg[b] = -min(r * adv[b], min(max(r, 1 - lo), 1 + hi) * adv[b])
        d[b] = 0.0 if off[b] else -adv[b] * r
        if ref is not None:
            q = ref[b] - lp[b]
            kl[b] = math.expm1(q) - q
            d[b] -= beta * math.expm1(q)
    share = w / sw if sw else w
    stats = [(share * x).sum() for x in (pg + beta * kl, pg, kl, off)]
    return stats, share * d


def ref_dz(p, labels, coef):
    dz = -p * coef
    dz[labels.clip(0, p.shape[0] - 1), np.arange(p.shape[1])] += coef
    return np.where(coef == 0, 0.0, dz)


def check_dz(got, p, labels, coef, scale, C, lp, dtype):
    """scale: the coefficients' scale that their error is relative to."""
    want = ref_dz(p, labels, coef)
    got = got.detach().cpu().double().numpy()
    with np.errstate(divide="ignore"):
        ep = es(C) + (np.abs(np.log(np.maximum(p, 1e-300))) + 4) * 2.0 ** -22
    own = np.zeros_like(p)
    own[labels.clip(0, C - 1), np.arange(p.shape[1])] = 1.0
    size = np.abs(own - p)
    tol = size * scale * 4 * (el(C, lp) + 2.0 ** -22) + np.abs(coef) * (p * ep + own * el(C, lp))
    tol = tol + np.abs(want) * HALF_STEP[dtype] * 1.001 + TINY[dtype]
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])
    assert not got[:, coef == 0].any()


SHAPES = [(1, 1), (2, 1), (10, 128), (7, 3), (10, 9), (33, 8), (100, 65), (257, 7), (1000, 333), (4097, 130), (5000, 1),
          (50257, 5), (64, 2051), (9, 9000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B", SHAPES)
def test_token_logp(C, B, dtype):
    z, labels, z64, lab = logits(C, B, dtype, seed=C + B)
    lp, _ = ref_logp(z64, lab, np.ones(B, bool))
    got = h(L1.token_logp(z, labels)).astype(np.float64)
    assert (np.abs(got - lp) <= el(C, lp)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B,pad,off", [(1, 1, 0, 0), (10, 128, 0, 0), (7, 3, 2, 1), (33, 8, 3, 5), (257, 7, 0, 0),
                                         (1000, 333, 1, 3), (4097, 130, 6, 0), (20, 2051, 0, 1), (50257, 5, 0, 0)])
@pytest.mark.parametrize("kl", [False, True])
def test_policy_loss(C, B, pad, off, dtype, kl):
    torch = _torch()
    z, labels, z64, lab = logits(C, B, dtype, seed=3 * C + B, pad=pad, off=off)
    rng = np.random.default_rng(B)
    w = np.where(rng.random(B) < 0.3, 0.0, rng.uniform(0.5, 2.0, B)).astype(np.float32)
    w[B // 2] = 1.0
    lab = lab.copy()
    lab[rng.random(B) < 0.1] = -100  # ignored
    lab[B // 2] = C - 1
    labels.copy_(torch.from_numpy(lab.astype(np.int32)))
    counts = (w != 0) & (lab >= 0)
    z[:, torch.from_numpy(~counts).to(z.device)] = float("nan")  # whatever the others hold
    lp, p = ref_logp(z64, lab, counts)
    step = 0.3 * rng.standard_normal(B)
    for border in (math.log(0.8), math.log(1.3)):  # no ratio where one rounding decides
        step = np.where(np.abs(step - border) < 0.02, border + 0.03, step)
    old, adv = (lp - step).astype(np.float32), rng.standard_normal(B).astype(np.float32)
    old[~counts], adv[~counts] = np.nan, np.inf
    ref = (lp + 0.5 * rng.standard_normal(B)).astype(np.float32) if kl else None
    stats, coef = ref_policy(lp, counts, w.astype(np.float64), old.astype(np.float64), adv.astype(np.float64),
                             None if ref is None else ref.astype(np.float64), 0.2, 0.3, 0.1)
    dbuf = torch.full((C, B + pad + 3), 7.0, dtype=z.dtype, device=z.device)
    st, dz, got = L1.policy_loss(z, labels, vec(old), vec(adv), ref_logp=None if ref is None else vec(ref), weights=vec(w),
                                 clip_low=0.2, clip_high=0.3, kl_coef=0.1, dlogits=dbuf[:, :B])
    assert (np.abs(h(got).astype(np.float64) - lp) <= el(C, lp)).all()
    share = np.where(counts, w, 0) / w[counts].sum()
    size = np.where(counts, np.exp(np.clip(lp - np.nan_to_num(old), -9, 9)) * np.abs(np.nan_to_num(adv, posinf=0)), 0)
    if kl:
        size = size + np.where(counts, 0.1 * (np.abs(np.expm1(ref - lp)) + 1), 0)
    # a mean's error: its terms' (1 + |q| for the kl, whose parts cancel), and one rounding
    tol = (share * (size + 3) * 4 * (el(C, lp) + 2.0 ** -22)).sum() + 2.0 ** -22 * (1 + np.abs(stats))
    assert (np.abs(h(st).astype(np.float64) - stats) <= tol).all(), (h(st), stats)
    check_dz(dz, p, lab, coef, share * size, C, lp, dtype)
    assert bool((dbuf[:, B:] == 7).all())  # the padding is not touched


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B,pairs", [(1, 4, 1), (10, 40, 3), (1000, 333, 4), (257, 7, 2), (300, 600, 100)])
@pytest.mark.parametrize("smoothing", [0.0, 0.2])
def test_preference_loss(C, B, pairs, dtype, smoothing):
    torch = _torch()
    z, labels, z64, lab = logits(C, B, dtype, seed=C * B)
    rng = np.random.default_rng(pairs)
    w = (rng.random(B) < 0.8).astype(np.float32)
    # empty sequences among them; tokens before the first and behind the last
    ptr = np.sort(rng.integers(1 if B > 8 else 0, B - B // 8 + 1, 2 * pairs + 1)).astype(np.int32)
    ptr[1] = ptr[0]
    inside = (np.arange(B) >= ptr[0]) & (np.arange(B) < ptr[-1])
    lp, p = ref_logp(z64, lab, w != 0)
    beta = 0.1
    sums = np.array([(w * lp)[ptr[q]:ptr[q + 1]].sum() for q in range(2 * pairs)])
    ref = (sums + rng.standard_normal(2 * pairs) * 5).astype(np.float32)
    rew = beta * (sums - ref.astype(np.float64))
    D = rew[0::2] - rew[1::2]
    ls = lambda x: -np.logaddexp(0, -x)  # noqa: E731
    sig = lambda x: 1 / (1 + np.exp(-x))  # noqa: E731
    loss = (-(1 - smoothing) * ls(D) - smoothing * ls(-D)).mean()
    dD = beta / pairs * (sig(D) - (1 - smoothing))
    coef = np.zeros(B)
    for q in range(2 * pairs):
        coef[ptr[q]:ptr[q + 1]] = (dD[q // 2] if q % 2 == 0 else -dD[q // 2]) * w[ptr[q]:ptr[q + 1]]
    dz = torch.full_like(z, 7.0)
    lo, dz, got = L1.preference_loss(z, labels, torch.from_numpy(ptr).to(z.device), ref_logp=vec(ref), weights=vec(w),
                                     beta=beta, label_smoothing=smoothing, dlogits=dz)
    err = np.array([(w * el(C, lp))[ptr[q]:ptr[q + 1]].sum() for q in range(2 * pairs)])
    assert (np.abs(h(got).astype(np.float64) - rew) <= beta * (err + 2.0 ** -23 * np.abs(sums)) + 2.0 ** -23 * np.abs(rew)).all()
    eD = beta * (err[0::2] + err[1::2])
    assert abs(float(lo) - loss) <= eD.max() + 2.0 ** -22 * (1 + abs(loss))  # |d loss / d D| <= 1
    scale = np.zeros(B)
    for q in range(2 * pairs):
        scale[ptr[q]:ptr[q + 1]] = beta / pairs * w[ptr[q]:ptr[q + 1]] * (1 + (err[q] + err[q ^ 1]) * beta / 4 / el(C, 0.0))
    check_dz(dz, p, lab, coef, scale, C, lp, dtype)
    assert not bool(dz[:, torch.from_numpy(~inside).to(z.device)].any())


def test_gradients_against_differences():
    # central differences of the losses' own values: step 2^-4, third derivatives below 1 (a loss of softmax probabilities
    # with |adv| <= 1, ratios near 1), so the truncation is below 2^-8 / 6 and the values' rounding 2^-22 / 2^-4
    torch = _torch()
    C, B = 11, 6
    z, labels, z64, lab = logits(C, B, "float32", seed=5)
    lp, _ = ref_logp(z64, lab, np.ones(B, bool))
    old, adv, ref = vec(lp - 0.05), vec(np.linspace(-1, 1, B)), vec(lp + 0.2)
    ptr = torch.tensor([0, 2, 3, 5, 6], dtype=torch.int32, device=z.device)
    policy = lambda x, g: L1.policy_loss(x, labels, old, adv, ref_logp=ref, kl_coef=0.5, clip_low=0.9, clip_high=9.0, grad=g)  # noqa: E731
    prefer = lambda x, g: L1.preference_loss(x, labels, ptr, beta=0.5, label_smoothing=0.1, grad=g)  # noqa: E731
    for f in (policy, prefer):
        dz = h(f(z, True)[1])
        step = 2.0 ** -4
        for c, b in ((0, 0), (3, 1), (int(lab[2]), 2), (10, 3), (int(lab[4]), 4), (5, 5)):
            v = []
            for s in (step, -step):
                x = z.clone()
                x[c, b] += s
                v.append(float(f(x, False)[0][0]))
            assert abs((v[0] - v[1]) / (2 * step) - dz[c, b]) <= step * step / 6 + 2.0 ** -22 / step, (c, b)


def test_masked_classes_and_empty_batches():
    torch = _torch()
    z, labels, z64, lab = logits(50, 12, "float32", seed=9)
    z[20:, ::2] = float("-inf")  # classes excluded; whole ranges of them
    lab = np.minimum(lab, 19)
    labels = torch.from_numpy(lab.astype(np.int32)).to(z.device)
    z[:, 3] = torch.finfo(torch.float32).min  # the type's lowest value everywhere: uniform
    z64 = z.cpu().double().numpy()
    with np.errstate(invalid="ignore"):
        lp, p = ref_logp(z64, lab, np.ones(12, bool))
    got = h(L1.token_logp(z, labels)).astype(np.float64)
    assert abs(got[3] + math.log(50)) <= el(50, lp[3])
    assert (np.abs(got - lp) <= el(50, lp)).all()
    st, dz, _ = L1.policy_loss(z, labels, vec(lp), vec(np.ones(12)))
    assert not bool(dz[20:, ::2].any()) and bool(torch.isfinite(dz).all())
    # no token counts: zeros
    st, dz, got = L1.policy_loss(z, labels, vec(lp), vec(np.ones(12)), weights=vec(np.zeros(12)))
    assert not bool(st.any()) and not bool(dz.any()) and not bool(got.any())
    # no tokens, no pairs
    e = torch.empty((50, 0), device=z.device)
    none = torch.empty(0, device=z.device)
    nolab = torch.empty(0, dtype=torch.int32, device=z.device)
    st, dz, got = L1.policy_loss(e, nolab, none, none)
    assert not bool(st.any()) and dz.shape == (50, 0) and got.numel() == 0
    assert L1.token_logp(e, nolab).numel() == 0
    loss, dz, rew = L1.preference_loss(z, labels, torch.zeros(1, dtype=torch.int32, device=z.device))
    assert float(loss) == 0.0 and not bool(dz.any()) and rew.numel() == 0
    loss, _, rew = L1.preference_loss(e, nolab, torch.zeros(3, dtype=torch.int32, device=z.device), ref_logp=vec([1.0, 2.0]))
    assert h(rew) == pytest.approx([-0.1, -0.2]) and float(loss) == pytest.approx(math.log1p(math.exp(-0.1)))


def test_offsets_outside_the_tokens_stay_in_bounds():
    # offsets beyond [0, B] or falling back are read as clamped ones: no token outside, no write outside dlogits
    torch = _torch()
    z, labels, _, _ = logits(20, 16, "float32", seed=2)
    bad = torch.tensor([-5, 4, 2, 99, 7], dtype=torch.int32, device=z.device)
    good = torch.tensor([0, 4, 4, 16, 16], dtype=torch.int32, device=z.device)
    first = torch.tensor([0, 4, 4], dtype=torch.int32, device=z.device)
    _, _, r = L1.preference_loss(z, labels, bad)
    _, _, want = L1.preference_loss(z, labels, first)
    assert h(r)[:2].tolist() == h(want).tolist()
    assert bool(torch.isfinite(r).all()) and good.numel() == 5


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_in_place_and_repeatable(dtype):
    torch = _torch()
    z, labels, _, _ = logits(700, 77, dtype, seed=1)
    old, adv = vec(np.full(77, -5.0)), vec(np.linspace(-1, 1, 77))
    st, dz, lp = L1.policy_loss(z, labels, old, adv)
    st2, dz2, lp2 = L1.policy_loss(z.clone(), labels, old, adv)
    assert torch.equal(dz, dz2) and torch.equal(st, st2) and torch.equal(lp, lp2)
    own = z.clone()
    _, back, _ = L1.policy_loss(own, labels, old, adv, dlogits=own)
    assert back is own and torch.equal(own, dz)
    ptr = torch.tensor([0, 30, 77], dtype=torch.int32, device=z.device)
    a = L1.preference_loss(z, labels, ptr)
    own = z.clone()
    b = L1.preference_loss(own, labels, ptr, dlogits=own)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    only = L1.policy_loss(z, labels, old, adv, grad=False)
    assert only[1] is None and torch.equal(only[0], st)


def test_streams_and_graphs():
    torch = _torch()
    z, labels, _, _ = logits(300, 129, "bfloat16", seed=4)
    old, adv = vec(np.full(129, -4.0)), vec(np.linspace(-1, 1, 129))
    ptr = torch.tensor([0, 60, 129], dtype=torch.int32, device=z.device)
    want = [L1.policy_loss(z, labels, old, adv), L1.preference_loss(z, labels, ptr)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [L1.policy_loss(z, labels, old, adv, stream=side), L1.preference_loss(z, labels, ptr, stream=side)]
    side.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    # two graphs captured one after the other, replayed beside each other with other inputs between
    zs, graphs, outs = [z.clone(), z.clone()], [], []
    for x in zs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((L1.policy_loss(x, labels, old, adv), L1.preference_loss(x, labels, ptr)))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(3):
        for i, x in enumerate(zs):
            x.copy_(torch.randn(300, 129, device=z.device) * (1 + i + k))
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for x, o in zip(zs, outs):
            for a, b in zip(o, (L1.policy_loss(x, labels, old, adv), L1.preference_loss(x, labels, ptr))):
                assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("B", [7, 300])
def test_offsets_past_32_bits(B):
    """Rows so far apart that offsets pass 2^32 elements: the bits of the same columns side by side."""
    torch = _torch()
    C, ld = 70001, 65537
    wide = torch.empty((C, ld), dtype=torch.bfloat16, device="cuda")
    z = wide[:, 11:11 + B]
    z.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    labels = torch.randint(0, C, (B,), device="cuda").to(torch.int32)
    labels[0] = C - 1
    old, adv = torch.full((B,), -11.0, device="cuda"), torch.linspace(-1, 1, B, device="cuda")
    near = z.contiguous()
    want = L1.policy_loss(near, labels, old, adv, dlogits=near)
    got = L1.policy_loss(z, labels, old, adv, dlogits=z)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_outputs_that_are_inputs_are_refused():
    torch = _torch()
    z = torch.randn((9, 40), device="cuda")
    labels = torch.zeros(40, dtype=torch.int32, device="cuda")
    old, adv, ref = (torch.randn(40, device="cuda") for _ in range(3))
    ptr = torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda")
    for kw in (dict(logp=old), dict(logp=adv), dict(logp=ref), dict(stats=old[:4]), dict(logp=z[0]),
               dict(logp=labels.view(torch.float32))):
        with pytest.raises(L1.L1CSRError):
            L1.policy_loss(z, labels, old, adv, ref_logp=ref, **kw)
    with pytest.raises(L1.L1CSRError):
        r = torch.zeros(2, device="cuda")
        L1.preference_loss(z, labels, ptr, ref_logp=r, rewards=r)


def test_refusals():
    torch = _torch()
    z, labels, _, _ = logits(20, 16, "float32", seed=2)
    old = vec(np.zeros(16))
    with pytest.raises(ValueError):
        L1.token_logp(z.t(), labels)
    with pytest.raises(ValueError):
        L1.token_logp(z, labels[:8])
    with pytest.raises(TypeError):
        L1.token_logp(z, labels.long())
    with pytest.raises(TypeError):
        L1.token_logp(z.double(), labels)
    with pytest.raises(ValueError):
        L1.policy_loss(z, labels, old[:4], old)
    with pytest.raises(ValueError):
        L1.policy_loss(z, labels, old, old, dlogits=torch.empty(20, 15, device=z.device))
    with pytest.raises(ValueError):
        L1.policy_loss(z, labels, old, old, dlogits=torch.empty_like(z).to(torch.bfloat16))
    with pytest.raises(ValueError):
        L1.policy_loss(z, labels, old, old, dlogits=z, grad=False)
    with pytest.raises(L1.L1CSRError):  # overlapping, not the same matrix
        buf = torch.zeros(21, 16, device=z.device)
        L1.policy_loss(buf[:20], labels, old, old, dlogits=buf[1:])
    with pytest.raises(L1.L1CSRError):
        L1.policy_loss(z, labels, old, old, clip_low=1.5)
    with pytest.raises(L1.L1CSRError):
        L1.policy_loss(z, labels, old, old, kl_coef=float("nan"))
    with pytest.raises(ValueError):
        L1.preference_loss(z, labels, torch.zeros(4, dtype=torch.int32, device=z.device))
    with pytest.raises(L1.L1CSRError):
        L1.preference_loss(z, labels, torch.zeros(3, dtype=torch.int32, device=z.device), label_smoothing=0.7)
    with pytest.raises(ValueError):
        L1.token_logp(z, labels.cpu())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B", [(9, 13), (700, 77), (4000, 3)])
def test_gradient_beside_the_logits(C, B, dtype):
    # logits and gradient as columns of one buffer: the bits of matrices apart, the other columns untouched
    torch = _torch()
    z, labels, _, _ = logits(C, B, dtype, seed=6)
    buf = torch.full((C, 3 * B + 1), 7.0, dtype=z.dtype, device=z.device)
    own, dz = buf[:, :B], buf[:, B:2 * B]
    own.copy_(z)
    old, adv = vec(np.full(B, -4.0)), vec(np.linspace(-1, 1, B))
    ptr = torch.tensor([0, B // 2, B], dtype=torch.int32, device=z.device)
    for f in (lambda x, d: L1.policy_loss(x, labels, old, adv, dlogits=d), lambda x, d: L1.preference_loss(x, labels, ptr, dlogits=d)):
        want = f(z, None)
        got = f(own, dz)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(own, z) and bool((buf[:, 2 * B:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B", [(10, 100), (32768, 64), (50257, 5)])
def test_scaled_gradients(C, B, dtype):
    """grad_scale comes before the one rounding of dlogits: what fp16 cannot hold of a mean's gradient over a large vocabulary
    (entries under 2^-24) is there in the scaled one, to the formula's tolerance."""
    torch = _torch()
    z, labels, z64, lab = logits(C, B, dtype, seed=8)
    lp, p = ref_logp(z64, lab, np.ones(B, bool))
    old, adv = (lp - 0.1).astype(np.float32), np.linspace(0.25, 1, B).astype(np.float32)
    ones = np.ones(B)
    _, coef = ref_policy(lp, ones.astype(bool), ones, old.astype(np.float64), adv.astype(np.float64), None, 0.2, 0.3, 0.0)
    size = np.exp(lp - old) * adv / B
    ptr = torch.tensor([0, B // 2, B], dtype=torch.int32, device=z.device)
    sums = np.array([lp[:B // 2].sum(), lp[B // 2:].sum()])
    slope = 0.1 * (1 / (1 + math.exp(-0.1 * (sums[0] - sums[1]))) - 1)
    pair = np.where(np.arange(B) < B // 2, slope, -slope)
    err = 0.1 / 4 * el(C, lp).sum() / el(C, 0.0)  # of the slope, in the coefficients' own unit
    policy = lambda **kw: L1.policy_loss(z, labels, vec(old), vec(adv), clip_high=0.3, **kw)  # noqa: E731
    prefer = lambda **kw: L1.preference_loss(z, labels, ptr, beta=0.1, **kw)  # noqa: E731
    for f, want, scale in ((policy, coef, size), (prefer, pair, 0.1 * (1 + err) * ones)):
        plain = f()
        for s in (2.0 ** 12, 0.3, -4.0):
            got = f(grad_scale=s)
            assert torch.equal(got[0], plain[0]) and torch.equal(got[2], plain[2])  # the loss and the log-probabilities are not scaled
            s32 = float(np.float32(s))
            check_dz(got[1], p, lab, want * s32, scale * abs(s32), C, lp, dtype)
        assert torch.equal(f(grad_scale=1.0)[1], plain[1]) and not bool(f(grad_scale=0.0)[1].any())
        if dtype == "float32":
            assert torch.equal(f(grad_scale=2.0 ** 12)[1], plain[1] * 2.0 ** 12)  # a power of two changes no bit
        if dtype == "float16" and C == 32768:
            lost = float((plain[1] == 0).float().mean())
            kept = float((f(grad_scale=2.0 ** 12)[1] == 0).float().mean())
            assert lost > 0.1 and kept < lost / 10
    for bad in (float("nan"), float("inf")):
        for f in (policy, prefer):
            with pytest.raises(L1.L1CSRError):
                f(grad_scale=bad)


# few tokens of a large vocabulary: a column at a time (fewer columns than a vector has values), many ranges of classes
FEW = [(50257, 1), (50257, 3), (131072, 1), (131071, 3), (40001, 2), (131072, 7)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B", FEW)
def test_few_tokens_count_every_class_once(C, B, dtype):
    """Equal logits: every exponential is 1 and their sum the integer C, exact in fp32 (below 2^24) in any order, so lp is
    -log C but for the logarithm's and one subtraction's rounding, 2^-22 (1 + log C) < 3.1e-6.  A class left out or counted
    twice moves it by 1 / C >= 7.6e-6.  Another class a token, raised by 20: its own place in the sum."""
    torch = _torch()
    labels = torch.full((B,), C // 2, dtype=torch.int32, device="cuda")
    z = torch.empty((C, B), dtype=getattr(torch, dtype), device="cuda")
    z[:] = torch.tensor([-3.0, 0.0, 5.0, 1.0, 2.0, 64.0, -64.0][:B], device="cuda")
    tol = 2.0 ** -22 * (1 + math.log(C))
    lp = h(L1.token_logp(z, labels)).astype(np.float64)
    assert (np.abs(lp + math.log(C)) <= tol).all()
    old, adv = vec(lp), vec(np.ones(B))
    st, dz, _ = L1.policy_loss(z, labels, old, adv, grad_scale=2.0 ** 10)
    # dz = 2^10 / B (1 / C - [c = a]): the ratio and 1 / C are within tol, dz rounds once
    want = np.full(C, 1.0 / C)
    want[C // 2] -= 1
    want *= 2.0 ** 10 / B
    err = np.abs(want) * (4 * tol + HALF_STEP[dtype]) + TINY[dtype]
    assert (np.abs(dz.cpu().double().numpy() - want[:, None]) <= err[:, None]).all()
    # one class far above the others: e^20 of the sum
    for c in (0, 1, 255, 256, 2010, 2011, C // 3, C - 257, C - 256, C - 2, C - 1):
        x = z.clone()
        x[c] += 20
        x64 = x.double()  # (the raised value as its type holds it)
        raised = (x64[c] - x64[C // 2]).cpu().numpy()
        S = np.exp(raised) + C - 1
        got = h(L1.token_logp(x, labels)).astype(np.float64)
        assert (np.abs(got + np.log(S)) <= el(512, np.log(S))).all(), c


def check_dz_of_depth(got, p, labels, coef, scale, depth, lp, dtype):
    """check_dz with the sums' error that of `depth` terms, whatever the number of classes."""
    C, B = p.shape
    want = ref_dz(p, labels, coef)
    got = got.detach().cpu().double().numpy()
    with np.errstate(divide="ignore"):
        ep = es(depth) + (np.abs(np.log(np.maximum(p, 1e-300))) + 4) * 2.0 ** -22
    own = np.zeros_like(p)
    own[labels, np.arange(B)] = 1.0
    tol = np.abs(own - p) * scale * 4 * (el(depth, lp) + 2.0 ** -22) + np.abs(coef) * (p * ep + own * el(depth, lp))
    tol = tol + np.abs(want) * HALF_STEP[dtype] * 1.001 + TINY[dtype]
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B", FEW)
def test_few_tokens_of_a_large_vocabulary(C, B, dtype):
    """Against the formula, with a sum's real depth: 8 rows at a time in a thread, at most 256 threads and 64 ranges joined."""
    torch = _torch()
    z, labels, z64, lab = logits(C, B, dtype, seed=C - B, pad=1)
    every = np.ones(B, bool)
    lp, p = ref_logp(z64, lab, every)
    tol = el(256, lp)  # (2 * 256 + 16) 2^-24
    assert (np.abs(h(L1.token_logp(z, labels)).astype(np.float64) - lp) <= tol).all()
    old, adv = (lp - 0.05).astype(np.float32), np.linspace(-1, 1, B).astype(np.float32) + 0.125
    ref = (lp + 0.3).astype(np.float32)
    stats, coef = ref_policy(lp, every, np.ones(B), old.astype(np.float64), adv.astype(np.float64), ref.astype(np.float64), 0.2,
                             0.3, 0.1)
    st, dz, got = L1.policy_loss(z, labels, vec(old), vec(adv), ref_logp=vec(ref), kl_coef=0.1, clip_high=0.3, grad_scale=256.0)
    assert (np.abs(h(got).astype(np.float64) - lp) <= tol).all()
    assert (np.abs(h(st).astype(np.float64) - stats) <= 16 * tol.max() + 2.0 ** -22 * (1 + np.abs(stats))).all()
    size = (np.exp(lp - old) * np.abs(adv) + 0.1 * (np.expm1(ref - lp) + 1)) / B
    check_dz_of_depth(dz, p, lab, coef * 256, size * 256, 256, lp, dtype)
    ptr = torch.tensor([0, (B + 1) // 2, B], dtype=torch.int32, device=z.device)
    loss, dz, rew = L1.preference_loss(z, labels, ptr, beta=0.1, grad_scale=256.0)
    sums = np.array([lp[:(B + 1) // 2].sum(), lp[(B + 1) // 2:].sum()])
    D = 0.1 * (sums[0] - sums[1])
    assert (np.abs(h(rew).astype(np.float64) - 0.1 * sums) <= 0.1 * tol.sum() + 2.0 ** -22 * np.abs(0.1 * sums)).all()
    assert abs(float(loss) - np.logaddexp(0, -D)) <= 0.1 * tol.sum() + 2.0 ** -22 * (1 + abs(D))
    slope = 0.1 * (1 / (1 + math.exp(-D)) - 1)
    coef = np.where(np.arange(B) < (B + 1) // 2, slope, -slope)
    scale = 0.1 * (1 + 0.1 / 4 * tol.sum() / el(256, 0.0)) * np.ones(B)
    check_dz_of_depth(dz, p, lab, coef * 256, scale * 256, 256, lp, dtype)


@pytest.mark.parametrize("C,B", [(20, 16), (4099, 16), (3000, 40)])
def test_offsets_outside_the_tokens(C, B):
    """Offsets beyond [0, B] or falling back, through the one-workgroup kernel and the pair pass: a pair reads lo = seq[2p]
    clamped to [0, B], mid = seq[2p + 1] to [lo, B], hi = seq[2p + 2] to [mid, B]; nothing outside dlogits is written."""
    torch = _torch()
    z, labels, z64, lab = logits(C, B, "float32", seed=2)
    lp, _ = ref_logp(z64, lab, np.ones(B, bool))
    guard = torch.full((C + 2, B + 6), 7.0, device=z.device)
    dz = guard[1:-1, 3:-3]
    big = 2 ** 31 - 1
    for bad in ([-5, 4, 2, 99, 7], [big, -big, big, 0, -1], [3, 1, -4, -9, big], [-big, big, -big, 5, 9]):
        _, _, rew = L1.preference_loss(z, labels, torch.tensor(bad, dtype=torch.int32, device=z.device), beta=0.5, dlogits=dz)
        want, err = [], []
        inside = np.zeros(B, bool)
        for q in range(2):
            lo = min(max(bad[2 * q], 0), B)
            mid = min(max(bad[2 * q + 1], lo), B)
            hi = min(max(bad[2 * q + 2], mid), B)
            want += [0.5 * lp[lo:mid].sum(), 0.5 * lp[mid:hi].sum()]
            err += [0.5 * el(C, lp)[lo:mid].sum(), 0.5 * el(C, lp)[mid:hi].sum()]
            inside[lo:hi] = True
        want = np.array(want)
        assert (np.abs(h(rew).astype(np.float64) - want) <= np.array(err) + 2.0 ** -22 * np.abs(want)).all(), bad
        assert bool(torch.isfinite(dz).all()) and not bool(dz[:, torch.from_numpy(~inside).to(z.device)].any())
        edge = guard.clone()
        edge[1:-1, 3:-3] = 7.0
        assert bool((edge == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,B", [(10, 64), (1000, 64)])
@pytest.mark.parametrize("e", [-131, -120, 122, 126])
def test_weights_of_any_size(C, B, e, dtype):
    """Weights enter by their shares: all of them times 2^e changes nothing, also where their sum's inverse is no normal float.
    (At 2^-131 the weights themselves hold 18 bits or more, their products with a gradient of 2^-2 or more 16: 2^-17 off.)"""
    torch = _torch()
    z, labels, z64, lab = logits(C, B, dtype, seed=12)
    lp, p = ref_logp(z64, lab, np.ones(B, bool))
    old = vec(lp - 0.05)
    adv = vec(np.linspace(0.5, 1, B) * np.where(np.arange(B) % 2, 1, -1))
    w = np.linspace(1, 1.9, B).astype(np.float32)
    w[::5] = 0
    st, dz, _ = L1.policy_loss(z, labels, old, adv, weights=vec(w), clip_high=0.3)
    st2, dz2, _ = L1.policy_loss(z, labels, old, adv, weights=vec(np.ldexp(w, e)), clip_high=0.3)
    assert not bool(dz2[:, ::5].any()) and bool(dz[:, 1::5].any())
    tol = 2.0 ** -17 if e == -131 else 2.0 ** -21  # (a few roundings of 2^-24)
    a, b = dz.cpu().double().numpy(), dz2.cpu().double().numpy()
    # both round to the type: half a step each, beside the weights'
    assert (np.abs(a - b) <= np.abs(a) * (tol + 2.002 * HALF_STEP[dtype]) + 2 * TINY[dtype]).all()
    assert (np.abs(h(st) - h(st2)) <= tol * (1 + np.abs(h(st)))).all()
    # a factor that only the products can hold
    st3, dz3, _ = L1.policy_loss(z, labels, old, adv, weights=vec(np.ldexp(w, e)), clip_high=0.3, grad_scale=2.0 ** 10)
    c = dz3.cpu().double().numpy() / 2.0 ** 10
    assert (np.abs(a - c) <= np.abs(a) * (tol + 2.002 * HALF_STEP[dtype]) + 2 * TINY[dtype]).all() and not dz3[:, ::5].any()
