"""What a fine-tuning step needs at its two ends, as cases that can be timed and compared: the losses on token
log-probabilities with their gradients (clipped policy loss with a KL term, preference loss over pairs of sequences, the
log-probabilities alone) and the update by orthogonalised momentum (Muon) with its proximal step.

Kinds of case

logp        log-probabilities of the taken tokens, logits[C][B] (classes by tokens): what scoring and serving call
policy      clipped policy loss and its gradient with respect to the logits
preference  preference loss over (chosen, rejected) sequences packed along the tokens, and its gradient
ortho       a matrix orthogonalised by five Newton-Schulz steps
muon        one Prox-Muon step of a CSR layer: momentum, orthogonalised update, soft threshold; the dense result

Layer sizes are those of the 784-300-100-10 MLP, the 4096 x 4096 layer and the 9216 -> 4096 layer; vocabularies and token counts
are generic.  Logits are what a trained head gives: N(0, 2) with the taken token raised by some units.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
A5, B5, C5 = 3.4445, -4.7750, 2.0315  # the quintic of the Newton-Schulz step: a x + b x^3 + c x^5
STEPS, EPS = 5, 1e-7
MU, ETA, LAM = 0.95, 0.02, 0.005
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
BETA, SMOOTHING = 0.1, 0.1


def listed():
    return [
        # the middle layer of the small MLP: a chain of short products, launches decide
        dict(name="muon_100x300", kind="muon", N=100, K=300, density=0.20),
        # the layer of the density sweep, square
        dict(name="muon_4096x4096", kind="muon", N=4096, K=4096, density=0.05),
        # the largest layer
        dict(name="muon_4096x9216", kind="muon", N=4096, K=9216, density=0.09),
        # first layer of the MLP, more columns than rows
        dict(name="ortho_300x784_f32", kind="ortho", N=300, K=784, dtype="f32"),
        # odd sizes, more rows than columns, half precision
        dict(name="ortho_1777x1001_f16", kind="ortho", N=1777, K=1001, dtype="f16"),
        # a layer of a network kept in bf16
        dict(name="ortho_4096x4096_bf16", kind="ortho", N=4096, K=4096, dtype="bf16"),
        # single tokens of seven sequences being served, a large vocabulary
        dict(name="logp_131072x7_f32", kind="logp", C=131072, B=7, dtype="f32"),
        # the MLP's ten classes as actions
        dict(name="policy_10x128_f32", kind="policy", C=10, B=128, dtype="f32", kl=False, masked=0.0),
        # odd vocabulary and token count
        dict(name="policy_50257x1021_f32", kind="policy", C=50257, B=1021, dtype="f32", kl=True, masked=0.1),
        # a batch of rollouts, padded
        dict(name="policy_32768x8192_bf16", kind="policy", C=32768, B=8192, dtype="bf16", kl=True, masked=0.3),
        # a few short pairs on a small vocabulary
        dict(name="preference_1000x333_f32", kind="preference", C=1000, pairs=4, B=333, dtype="f32", masked=0.2),
        # a batch of pairs
        dict(name="preference_32768x4099_bf16", kind="preference", C=32768, pairs=8, B=4099, dtype="bf16", masked=0.4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("logp", "policy", "policy", "preference", "ortho", "muon", "muon"))
    if kind in ("ortho", "muon"):
        N, K = _log(rng, 10, 4096), _log(rng, 10, 9216)
        N = 2 * (N // 2) + rng.randrange(2)
        if kind == "muon":
            return dict(kind=kind, N=N, K=K, density=round(rng.uniform(0.02, 0.5), 2))
        return dict(kind=kind, N=N, K=K, dtype=rng.choice(("f32", "f32", "bf16", "f16")))
    C = _log(rng, 10, 131072)
    B = _log(rng, 8 if kind == "preference" else 1, min(8192, (1 << 28) // C))
    case = dict(kind=kind, C=C, B=B, dtype=rng.choice(("f32", "bf16", "bf16", "f16")))
    if kind == "logp":
        return case
    case["masked"] = round(rng.uniform(0.0, 0.5), 2)
    if kind == "policy":
        return dict(case, kl=rng.random() < 0.7)
    return dict(case, pairs=max(1, min(B // 4, _log(rng, 1, 64))))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _logits(case, g):
    """Logits of the case's type, and the taken tokens."""
    C, B = case["C"], case["B"]
    z = torch.randn((C, B), generator=g, device="cuda") * 2.0
    labels = torch.randint(0, C, (B,), generator=g, device="cuda")
    raised = torch.rand((B,), generator=g, device="cuda") * (2.0 + math.log(C))
    z[labels, torch.arange(B, device="cuda")] += raised
    return z.to(TYPES[case["dtype"]]), labels.to(torch.int32)


def _logp_of(z, labels):
    B = z.shape[1]
    z = z.float()
    top = z.amax(0)
    return z[labels.long(), torch.arange(B, device="cuda")] - top - (z - top).exp_().sum(0).log()


def _layer_grad(N, K, g):
    """What backpropagation leaves in a dense gradient: a few strong directions over noise."""
    strong = torch.randn((N, 4), generator=g, device="cuda") @ torch.rand((4, K), generator=g, device="cuda")
    return (0.02 * strong + 0.05 * torch.randn((N, K), generator=g, device="cuda")) * 1e-3


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=case)
    kind = case["kind"]
    if kind == "ortho":
        s["G"] = _layer_grad(case["N"], case["K"], g).to(TYPES[case["dtype"]])
        s["out"] = torch.empty_like(s["G"])
        return s
    if kind == "muon":
        N, K = case["N"], case["K"]
        dense = torch.randn((N, K), generator=g, device="cuda") * 0.05
        dense *= torch.rand((N, K), generator=g, device="cuda") < case["density"]
        kept = dense != 0
        s["row_ptr"] = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int64), kept.sum(1).cumsum(0)]).to(torch.int32)
        s["col_idx"] = kept.nonzero()[:, 1].to(torch.int32)
        s["vals"] = dense[kept]
        s["nnz"] = int(s["row_ptr"][-1])
        s["G"] = _layer_grad(N, K, g)
        s["m"] = _layer_grad(N, K, g) * 6.0
        s["m_out"] = torch.empty_like(s["m"])
        s["Z"] = torch.empty_like(s["m"])
        return s
    s["z"], s["labels"] = _logits(case, g)
    B = case["B"]
    if kind == "logp":
        s["logp"] = torch.empty(B, device="cuda")
        return s
    s["dz"] = torch.empty_like(s["z"])
    s["weights"] = (torch.rand((B,), generator=g, device="cuda") >= case["masked"]).float()
    s["weights"][B // 2] = 1.0
    lp = _logp_of(s["z"], s["labels"])
    if kind == "policy":
        # the policy moved a little since the rollout; no ratio within 1e-3 of a border of the clip, where one rounding
        # decides whether a token has a gradient
        step = 0.25 * torch.randn((B,), generator=g, device="cuda")
        for border in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
            near = (step - border).abs() < 1e-3
            step = torch.where(near, step + 4e-3, step)
        s["old_logp"] = lp - step
        s["adv"] = torch.randn((B,), generator=g, device="cuda")
        s["ref_logp"] = lp + 0.3 * torch.randn((B,), generator=g, device="cuda") if case["kl"] else None
        return s
    pairs = case["pairs"]
    cuts = torch.rand((2 * pairs - 1,), generator=g, device="cuda").sort().values
    inner = (cuts * (B - B // 16)).to(torch.int32)  # the last tokens pad the batch: in no sequence
    ends = torch.tensor([B - B // 16], dtype=torch.int32, device="cuda")
    s["seq_ptr"] = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), inner, ends])
    lens = (s["seq_ptr"][1:] - s["seq_ptr"][:-1]).double()
    total = torch.cat([torch.zeros(1, dtype=torch.float64, device="cuda"), (lp * s["weights"]).double().cumsum(0)])
    at = s["seq_ptr"].long()
    sums = total[at[1:]] - total[at[:-1]]
    s["ref_logp"] = (sums + lens.sqrt() * 0.5 * torch.randn((2 * pairs,), generator=g, device="cuda")).float()
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_1905_07931_amd as L1
    case = s["case"]
    kind = case["kind"]
    if kind == "ortho":
        return L1.orthogonalize(s["G"], out=s["out"])
    if kind == "muon":
        W = L1.CSR(case["N"], case["K"], s["row_ptr"], s["col_idx"], s["vals"], s["nnz"])
        st = L1.MuonState(s["m"], mu=MU, nesterov=True, steps=STEPS, eps=EPS)
        Z = L1.prox_muon_step(W, s["G"], st, ETA, LAM, Z=s["Z"], m_out=s["m_out"])
        return {"Z": Z, "m": s["m_out"]}
    if kind == "logp":
        return L1.token_logp(s["z"], s["labels"], logp=s["logp"])
    if kind == "policy":
        stats, dz, logp = L1.policy_loss(s["z"], s["labels"], s["old_logp"], s["adv"], ref_logp=s["ref_logp"],
                                         weights=s["weights"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                                         kl_coef=KL, dlogits=s["dz"])
        return {"stats": stats, "dz": dz, "logp": logp}
    loss, dz, rewards = L1.preference_loss(s["z"], s["labels"], s["seq_ptr"], ref_logp=s["ref_logp"],
                                           weights=s["weights"], beta=BETA, label_smoothing=SMOOTHING, dlogits=s["dz"])
    return {"loss": loss, "dz": dz, "rewards": rewards}


def _plain_newton_schulz(U):
    X = U.t() if U.shape[0] > U.shape[1] else U
    X = (X / (U.double().square().sum().sqrt() + EPS)).contiguous()
    for _ in range(STEPS):
        A = X @ X.t().contiguous()
        X = A5 * X + (B5 * A + C5 * (A @ A)) @ X
    return X.t() if U.shape[0] > U.shape[1] else X


def _plain_token(s):
    """(shifted exponentials, their sums, log-probabilities of the taken tokens)."""
    z, B = s["z"].float(), s["case"]["B"]
    z = z - z.amax(0)
    taken = z[s["labels"].long(), torch.arange(B, device="cuda")]
    e = z.exp()
    total = e.sum(0)
    return e, total, taken - total.log()


def _plain_gradient(s, coef, e, total):
    dz = e * (-coef / total)
    cols = torch.arange(coef.shape[0], device="cuda")
    dz[s["labels"].long(), cols] += coef
    return dz.to(s["z"].dtype)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "ortho":
        return _plain_newton_schulz(s["G"].float()).to(s["G"].dtype).contiguous()
    if kind == "muon":
        N, K = case["N"], case["K"]
        m = MU * s["m"] + s["G"]
        O = _plain_newton_schulz(s["G"] + MU * m) * math.sqrt(max(1.0, N / K))
        W = torch.zeros((N, K), device="cuda")
        rows = torch.repeat_interleave(torch.arange(N, device="cuda"), (s["row_ptr"][1:] - s["row_ptr"][:-1]).long(),
                                       output_size=s["nnz"])
        W[rows, s["col_idx"].long()] = s["vals"]
        Z = W - ETA * O
        return {"Z": Z.sign() * (Z.abs() - ETA * LAM).clamp_min(0.0), "m": m}
    e, total, lp = _plain_token(s)
    if kind == "logp":
        return lp
    w = s["weights"]
    if kind == "policy":
        sum_w = w.double().sum()
        r = (lp - s["old_logp"]).exp()
        adv = s["adv"]
        clipped = r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
        off = clipped < r * adv
        pg = -torch.minimum(r * adv, clipped)
        d = torch.where(off, torch.zeros_like(r), -adv * r)
        kl = torch.zeros_like(r)
        if s["ref_logp"] is not None:
            q = s["ref_logp"] - lp
            kl = q.exp() - q - 1
            d = d + KL * (1 - q.exp())
        mean = lambda x: ((w * x).double().sum() / sum_w)  # noqa: E731
        stats = torch.stack([mean(pg + KL * kl), mean(pg), mean(kl), mean(off.float())]).float()
        coef = (w * d / sum_w).float()
        return {"stats": stats, "dz": _plain_gradient(s, coef, e, total), "logp": lp * (w != 0)}
    P, B, ptr = case["pairs"], case["B"], s["seq_ptr"]
    of = torch.searchsorted(ptr, torch.arange(B, device="cuda", dtype=torch.int32), right=True) - 1
    inside = (of >= 0) & (of < 2 * P)
    w = w * inside
    of = of.clamp(0, 2 * P - 1)
    sums = torch.zeros(2 * P, dtype=torch.float64, device="cuda").index_add_(0, of, (w * lp).double())
    rewards = BETA * (sums - s["ref_logp"])
    D = rewards[0::2] - rewards[1::2]
    up, down = torch.sigmoid(D), torch.sigmoid(-D)
    loss = (-(1 - SMOOTHING) * down.neg().log1p() - SMOOTHING * up.neg().log1p()).mean()
    dD = (SMOOTHING * up - (1 - SMOOTHING) * down) * (BETA / P)
    coef = (torch.stack([dD, -dD], 1).reshape(-1)[of] * w).float()
    return {"loss": loss.float().reshape(1), "dz": _plain_gradient(s, coef, e, total), "rewards": rewards.float()}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it has to give
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("ortho", "muon"):
        m, n = sorted((case["N"], case["K"]))
        # A and the polynomial of A are symmetric (half a product each); several steps may share one product with X, the
        # polynomials of the steps between being m x m
        stepwise = STEPS * (3 * m * m * n + m ** 3)
        shared = 6 * m * m * n + 14 * m ** 3
        if kind == "ortho":
            return {"bytes": 2 * m * n * BYTES[case["dtype"]], "flops": min(stepwise, shared)}
        return {"bytes": 16 * m * n + 8 * case["density"] * m * n + 4 * case["N"], "flops": min(stepwise, shared)}
    n, e = case["C"] * case["B"], BYTES[case["dtype"]]
    if kind == "logp":
        return {"bytes": n * e + 8 * case["B"], "flops": 4 * n}
    return {"bytes": 2 * n * e + 24 * case["B"], "flops": 8 * n}


def _exact_newton_schulz(U):
    """By the powers of the smaller Gram matrix alone: with P_k = a + b A_k + c A_k^2 the result is ... P_2 P_1 P_0 X and
    A_(k+1) = P_k A_k P_k."""
    X = U / (torch.linalg.matrix_norm(U) + EPS)
    wide = X.shape[0] <= X.shape[1]
    A = X @ X.t().contiguous() if wide else X.t().contiguous() @ X
    one = torch.eye(A.shape[0], dtype=torch.float64, device=A.device)
    Q = one
    for _ in range(STEPS):
        P = A5 * one + A @ (B5 * one + C5 * A)
        Q, A = P @ Q, P @ A @ P
    return Q @ X if wide else X @ Q


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "ortho":
        return _exact_newton_schulz(s["G"].double())
    if kind == "muon":
        N, K = case["N"], case["K"]
        G, m0 = s["G"].double(), s["m"].double()
        m = G + MU * m0
        W = torch.sparse_csr_tensor(s["row_ptr"].long(), s["col_idx"].long(), s["vals"].double(), (N, K)).to_dense()
        Z = W - ETA * max(1.0, N / K) ** 0.5 * _exact_newton_schulz(G + MU * m)
        t = ETA * LAM
        return {"Z": (Z - t).clamp_min(0) + (Z + t).clamp_max(0), "m": m}
    z, labels = s["z"].double(), s["labels"].long()
    lse = torch.logsumexp(z, 0)
    lp = z.gather(0, labels[None]).squeeze(0) - lse
    if kind == "logp":
        return lp
    w = s["weights"].double()
    if kind == "policy":
        share = w / w.sum()
        adv, move = s["adv"].double(), lp - s["old_logp"].double()
        high, low = math.log1p(CLIP_HIGH), math.log1p(-CLIP_LOW)
        off = ((adv > 0) & (move > high)) | ((adv < 0) & (move < low))
        used = torch.where(off, move.clamp(low, high), move).exp()
        pg = -adv * used
        kl, dkl = torch.zeros_like(lp), torch.zeros_like(lp)
        if s["ref_logp"] is not None:
            q = s["ref_logp"].double() - lp
            kl, dkl = torch.expm1(q) - q, -torch.expm1(q)
        coef = share * (torch.where(off, 0.0, pg) + KL * dkl)
        stats = torch.stack([(share * x).sum() for x in (pg + KL * kl, pg, kl, off.double())])
        kept = torch.where(w != 0, lp, 0.0)
        return {"stats": stats, "dz": _exact_gradient(z, labels, lse, coef), "logp": kept}
    P, ptr = case["pairs"], s["seq_ptr"].tolist()
    rewards, coef = torch.zeros(2 * P, dtype=torch.float64, device="cuda"), torch.zeros_like(lp)
    for q in range(2 * P):
        a, b = ptr[q], ptr[q + 1]
        rewards[q] = BETA * ((w[a:b] * lp[a:b]).sum() - s["ref_logp"][q].double())
    D = rewards[0::2] - rewards[1::2]
    ls = torch.nn.functional.logsigmoid
    loss = -((1 - SMOOTHING) * ls(D) + SMOOTHING * ls(-D)).mean()
    slope = BETA / P * (torch.sigmoid(D) - (1 - SMOOTHING))
    for q in range(2 * P):
        a, b = ptr[q], ptr[q + 1]
        coef[a:b] = (slope[q // 2] if q % 2 == 0 else -slope[q // 2]) * w[a:b]
    return {"loss": loss.reshape(1), "dz": _exact_gradient(z, labels, lse, coef), "rewards": rewards}


def _exact_gradient(z, labels, lse, coef):
    dz = (z - lse).exp_().mul_(-coef)
    dz.scatter_add_(0, labels[None], coef[None])
    return dz
