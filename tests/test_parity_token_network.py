"""A training step of a small network on tokens, end to end, with the library's calls alone: embedding (a table kept in CSR, or
dense and tied to the output layer), norms with gate and residual around a compressed layer, logits, a loss, every gradient
back to the table, clipping of all of them together, the proximal step; against the same network in 64 bits with torch's
automatic gradients on the CPU.

Tolerances: every value passes through a handful of fp32 sums of at most 300 terms, each within 300 * 2^-24 = 1.8e-5 of its
size at worst; gradients are compared relative to their largest entry, 1e-4 as the library's products are.  One term is worse than that:
where a token's probability is near 1 its own logit's gradient is coef (p - 1) = coef expm1(lp), and lp is a difference
of logits and the logarithm of a sum of C exponentials, absolutely within EL = (2 C + 16) 2^-24 + 2^-22 (1 + |lp|) (one
rounding of the exponent, one of the exponential and two of the sum a class).  So that gradient is off by |coef| EL, and
a gradient of the network, which is linear in it, by |coef| EL |d z_own / d theta| for every token: the sum of these over the
tokens is added to the tolerance.  (Seed 7, token 35: ratio 57.7, lp near 0, coef 1.76; the same network in fp32 on the
CPU is 1.6e-3 off.)
"""
import numpy as np
import pytest

import paper_1905_07931_amd as L1

from _helpers import cuda

pytestmark = pytest.mark.gpu

V, D, B, N = 60, 48, 70, 48


def _torch():
    import torch
    return torch


def sparse(rng, n, k, density):
    torch = _torch()
    keep = rng.random((n, k)) < density
    dense = np.where(keep, rng.standard_normal((n, k)) * 0.3, 0).astype(np.float32)
    ptr = np.concatenate([[0], keep.sum(1).cumsum()]).astype(np.int32)
    W = L1.CSR(n, k, torch.from_numpy(ptr).to(cuda()), torch.from_numpy(np.nonzero(keep)[1].astype(np.int32)).to(cuda()),
               torch.from_numpy(dense[keep]).to(cuda()), int(ptr[-1]))
    return W, torch.from_numpy(dense).double(), torch.from_numpy(keep)


def close(got, want, what):
    """want: (gradient, what its entries may be off by beyond 1e-4 of the largest)"""
    want, slack = (x.detach().double() for x in want)
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    size, err = float(want.abs().max()), (got - want).abs()
    assert bool((err <= 1e-4 * size + slack).all()), (what, float((err - slack).max()), size)


def of(pair, f):
    """A function of a gradient, and of its slack."""
    return tuple(f(x) for x in pair)


def data(seed):
    torch = _torch()
    rng = np.random.default_rng(seed)
    tokens = rng.integers(0, V, B)
    tokens[rng.random(B) < 0.3] = 3  # a frequent one
    tokens[-5:] = -1                 # padding
    labels = rng.integers(0, V, B)
    weights = (tokens >= 0).astype(np.float32)
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))  # noqa: E731
    p = dict(pre=1 + 0.2 * f(D), post=0.6 + 0.2 * f(D), final=1 + 0.2 * f(D), gate=f(D, B), old=-4 + 0.2 * f(B), adv=f(B))
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).to(cuda())  # noqa: E731
    return rng, tokens, labels, i32(tokens), i32(labels), torch.from_numpy(weights).to(cuda()), p


def reference(table, tied, hidden, tokens, labels, p, scale):
    """Loss and gradients in 64 bits."""
    torch = _torch()
    leaves = dict(table=table.clone(), hidden=hidden.clone(), **{k: p[k].double() for k in ("pre", "post", "final", "gate")})
    for x in leaves.values():
        x.requires_grad_()
    head = leaves["table"] if tied is None else tied.clone().requires_grad_()
    norm = lambda x, g: x / (x.square().mean(0) + 1e-6).sqrt() * g[:, None]  # noqa: E731
    good = torch.from_numpy((tokens >= 0).astype(np.float64))
    X = leaves["table"][torch.from_numpy(np.maximum(tokens, 0))].t() * good * scale
    y = leaves["hidden"] @ norm(X, leaves["pre"])
    r = X + 0.5 * torch.sigmoid(leaves["gate"]) * norm(y, leaves["post"])
    logits = head @ norm(r, leaves["final"])
    lp = (logits - logits.logsumexp(0))[torch.from_numpy(labels), torch.arange(B)]
    ratio = (lp - p["old"].double()).exp()
    adv = p["adv"].double()
    pg = -torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv)
    loss = (pg * good).sum() / good.sum()
    names = [*leaves] + ([] if tied is None else ["head"])
    at = [*leaves.values()] + ([] if tied is None else [head])
    grads = torch.autograd.grad(loss, at, retain_graph=True)
    coef = torch.autograd.grad(loss, lp, retain_graph=True)[0].abs()
    el = (2 * V + 16) * 2.0 ** -24 + 2.0 ** -22 * (1 + lp.detach().abs())
    slack = [torch.zeros_like(x) for x in at]
    for b in torch.nonzero(coef)[:, 0].tolist():
        for s, g in zip(slack, torch.autograd.grad(logits[labels[b], b], at, retain_graph=True)):
            s += float(coef[b] * el[b]) * g.abs()
    return loss.detach(), dict(zip(names, zip(grads, slack)))


def forward_backward(d, hidden, embed, head_product, p, scale):
    """The device's pass up to the gradient of the embedding's columns; returns it with the other gradients."""
    dev = {k: p[k].to(cuda()) for k in p}
    X = embed()
    _, h1 = L1.residual_norm_fwd(X, pre_gain=dev["pre"])
    y = L1.csr_spmm_fwd(hidden, h1)
    kw = dict(gate=dev["gate"], post_gain=dev["post"], pre_gain=dev["final"], alpha=0.5, sigmoid=True)
    r, h2 = L1.residual_norm_fwd(X, y, **kw)
    logits = head_product(h2)
    stats, dz, _ = L1.policy_loss(logits, d["labels"], dev["old"], dev["adv"], weights=d["weights"], clip_low=0.2, clip_high=0.2)
    dh2, head_grad = d["head_bwd"](dz, h2)
    g2 = L1.residual_norm_bwd(r, None, dh2, y, **kw)
    dh1 = L1.csr_spmm_bwd_t(hidden, g2.y, L1.csc_build(hidden))
    g1 = L1.residual_norm_bwd(X, g2.r, dh1, pre_gain=dev["pre"])
    return stats, g1.r, head_grad, L1.dense_wgrad(g2.y, h1), dict(pre=g1.pre_gain, post=g2.post_gain, final=g2.pre_gain, gate=g2.gate)


@pytest.mark.parametrize("seed", [0, 1])
def test_compressed_table_and_head(seed):
    torch = _torch()
    rng, tokens, labels, t, lab, w, p = data(seed)
    table, table64, keep = sparse(rng, V, D, 0.5)
    hidden, hidden64, _ = sparse(rng, N, D, 0.4)
    head, head64, _ = sparse(rng, V, N, 0.5)
    scale = 2.0
    d = dict(labels=lab, weights=w, head_bwd=lambda dz, h: (L1.csr_spmm_bwd_t(head, dz, L1.csc_build(head)), L1.dense_wgrad(dz, h)))
    stats, dX, dhead, dhidden, rest = forward_backward(d, hidden, lambda: L1.embedding_fwd(table, t, scale=scale),
                                                       lambda h: L1.csr_spmm_fwd(head, h), p, scale)
    loss, want = reference(table64, head64, hidden64, tokens, labels, p, scale)
    assert abs(float(stats[0]) - float(loss)) <= 1e-4
    plan = L1.embedding_plan(t, V)
    dtable = L1.embedding_bwd(dX, None, V, scale=scale, plan=plan)
    masked = L1.embedding_masked_bwd(table, dX, None, scale=scale, plan=plan)
    close(dtable, want["table"], "table")
    close(masked, of(want["table"], lambda x: x[keep]), "table, masked")
    close(dhead, want["head"], "head")
    close(dhidden, want["hidden"], "hidden")
    for k in rest:
        close(rest[k], want[k], k)
    # all gradients clipped together, and the proximal step of the three compressed layers
    grads = [dtable, dhead, dhidden, *rest.values()]
    norm = float(torch.sqrt(sum((g ** 2).sum() for g, _ in want.values())))
    off = float(torch.sqrt(sum((s ** 2).sum() for _, s in want.values())))
    stats = L1.clip_grad_norm(grads, norm / 2)
    assert abs(float(stats[0]) - norm) <= 1e-4 * norm + off and abs(float(stats[1]) - 0.5) <= 1e-4 + off / norm
    close(dhidden, of(want["hidden"], lambda x: x / 2), "hidden, clipped")
    eta, lam = 0.5, 0.01
    W2 = L1.prox_l1_recompress(table, dtable, eta, lam)
    z = table64 - eta * 0.5 * want["table"][0]
    z = z.sign() * (z.abs() - eta * lam).clamp_min(0)
    got = torch.zeros(V, D, dtype=torch.float64)
    n = W2.host_nnz()
    rows = np.repeat(np.arange(V), np.diff(W2.row_ptr.cpu().numpy()))
    got[rows, W2.col_idx[:n].cpu().long()] = W2.vals[:n].cpu().double()
    assert float((got - z).abs().max()) <= 1e-4 * float(z.abs().max())


def test_tied_dense_table():
    """The table serves as output layer as well: its gradient is the layer's with the embedding's added in place."""
    torch = _torch()
    rng, tokens, labels, t, lab, w, p = data(7)
    hidden, hidden64, _ = sparse(rng, N, D, 0.4)
    E = torch.from_numpy((rng.standard_normal((V, D)) * 0.3).astype(np.float32)).to(cuda())
    full = L1.CSR(V, D, torch.arange(0, V * D + 1, D, dtype=torch.int32, device=cuda()),
                  torch.arange(D, dtype=torch.int32, device=cuda()).repeat(V), E.flatten(), V * D)  # the same numbers as a layer
    d = dict(labels=lab, weights=w, head_bwd=lambda dz, h: (L1.csr_spmm_bwd_t(full, dz, L1.csc_build(full)), L1.dense_wgrad(dz, h)))
    _, dX, dE, dhidden, rest = forward_backward(d, hidden, lambda: L1.embedding_fwd(E, t, scale=1.5),
                                                lambda h: L1.csr_spmm_fwd(full, h), p, 1.5)
    assert L1.embedding_bwd(dX, t, V, dE=dE, add=dE, scale=1.5) is dE
    _, want = reference(E.cpu().double(), None, hidden64, tokens, labels, p, 1.5)
    close(dE, want["table"], "table")
    close(dhidden, want["hidden"], "hidden")
    for k in rest:
        close(rest[k], want[k], k)


def test_a_step_captured_with_other_work_between():
    """The whole pass in a graph, replayed on new tokens, against the eager pass bit for bit."""
    torch = _torch()
    rng, tokens, labels, t, lab, w, p = data(3)
    table, _, _ = sparse(rng, V, D, 0.5)
    hidden, _, _ = sparse(rng, N, D, 0.4)
    head, _, _ = sparse(rng, V, N, 0.5)
    csc = [L1.csc_build(m) for m in (head, hidden)]
    dev = {k: p[k].to(cuda()) for k in p}
    kw = dict(gate=dev["gate"], post_gain=dev["post"], pre_gain=dev["final"], alpha=0.5, sigmoid=True)

    def step():
        X = L1.embedding_fwd(table, t, scale=2.0)
        _, h1 = L1.residual_norm_fwd(X, pre_gain=dev["pre"])
        y = L1.csr_spmm_fwd(hidden, h1)
        r, h2 = L1.residual_norm_fwd(X, y, **kw)
        stats, dz, _ = L1.policy_loss(L1.csr_spmm_fwd(head, h2), lab, dev["old"], dev["adv"], weights=w)
        g2 = L1.residual_norm_bwd(r, None, L1.csr_spmm_bwd_t(head, dz, csc[0]), y, **kw)
        g1 = L1.residual_norm_bwd(X, g2.r, L1.csr_spmm_bwd_t(hidden, g2.y, csc[1]), pre_gain=dev["pre"])
        out = [L1.embedding_bwd(g1.r, t, V, scale=2.0), L1.dense_wgrad(dz, h2), L1.dense_wgrad(g2.y, h1), g1.pre_gain,
               g2.pre_gain, g2.post_gain, g2.gate]
        return [L1.clip_grad_norm(out, 0.01, zero_nonfinite=True), stats, *out]
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        res = step()
    for turn in range(4):
        t.copy_(torch.from_numpy(np.random.default_rng(turn).integers(-1, V, B).astype(np.int32)))
        g.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in res]
        eager = step()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(kept, eager)):
            assert torch.equal(a, b), (turn, i)
