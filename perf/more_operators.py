"""What a network on tokens has around its compressed layers, as cases that can be timed and compared: the embedding with
its gradients, the norms between blocks with gate and residual, and the gradients' global norm with clipping.

Kinds of case

embed       X[d][b] = scale E[token b][d]: rows of a dense table as columns of the activations
embed_csr   the same from a table kept in CSR, like every other weight
embed_bwd   the table's dense gradient (every row of it), alone or added to another (a table tied to the output layer)
embed_mask  the table's gradient on the pattern of its CSR (debiasing)
norm        n = norm(y) post_gain, r' = r + alpha a(gate) n, h = norm(r') pre_gain; norm over the features of a token
norm_bwd    its gradients: residual, block output, gate, both gains
clip        global norm of many gradients; each times min(1, max_norm / (norm + eps)) / grad_scale

Activations are [features][tokens], tokens contiguous.  Layer sizes are those of the 784-300-100-10 MLP, LeNet-5, the
4096 x 4096 layer and the 9216 -> 4096 layer; vocabularies and token counts are generic.  Tokens follow Zipf's law, the last
sixteenth of a batch pads it (-1).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
MLP = "300x784,300,100x300,100,10x100,10"
BIG = ",".join(["4096x9216,4096,4096x4096,4096"] * 4)


def listed():
    return [
        # one sequence being served: the next token's column, latency decides
        dict(name="embed_4096x1_f32", kind="embed", V=32768, D=4096, B=1, dtype="f32", out="f32"),
        # a training batch, the table kept in bf16, the layers' activations in fp32
        dict(name="embed_4096x8192_bf16", kind="embed", V=131072, D=4096, B=8192, dtype="bf16", out="f32"),
        # a compressed table of an odd vocabulary, odd batch
        dict(name="embed_csr_4096x1021", kind="embed_csr", V=50257, D=4096, B=1021, density=0.05),
        # a training batch's dense gradient: what the l1 update of the table takes
        dict(name="embed_bwd_4096x8192_f32", kind="embed_bwd", V=32768, D=4096, B=8192, dtype="f32", out="f32", tied=False),
        # a table tied to the output layer: its gradient is the sum of both, the layer's own being kept; odd sizes
        dict(name="embed_bwd_tied_1001x1021_bf16", kind="embed_bwd", V=50257, D=1001, B=1021, dtype="bf16", out="f32", tied=True),
        # debiasing of a compressed table
        dict(name="embed_mask_1024x4096", kind="embed_mask", V=32768, D=1024, B=4096, density=0.09),
        # one token between two blocks
        dict(name="norm_4096x1_f32", kind="norm", K=4096, B=1, dtype="f32", gate="row", sigmoid=False, post=True),
        # a training batch between two blocks, each value gated
        dict(name="norm_4096x8192_bf16", kind="norm", K=4096, B=8192, dtype="bf16", gate="full", sigmoid=True, post=True),
        # odd sizes, a gain a feature as the gate
        dict(name="norm_bwd_1001x333_f32", kind="norm_bwd", K=1001, B=333, dtype="f32", gate="row", sigmoid=False, post=True),
        # the inputs of the largest layer
        dict(name="norm_bwd_9216x2048_f32", kind="norm_bwd", K=9216, B=2048, dtype="f32", gate="full", sigmoid=True, post=True),
        # the small MLP
        dict(name="clip_mlp_f32", kind="clip", layers=MLP, dtype="f32", out="f32", grad_scale=1.0, max_norm=1.0),
        # four blocks of the two large layers, the losses' scale in the gradients
        dict(name="clip_4096_bf16", kind="clip", layers=BIG, dtype="bf16", out="f32", grad_scale=1024.0, max_norm=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("embed", "embed_csr", "embed_bwd", "embed_bwd", "embed_mask", "norm", "norm", "norm_bwd", "norm_bwd",
                       "clip"))
    if kind.startswith("embed"):
        D = _log(rng, 10, 4096)
        V = _log(rng, 10, min(131072, (1 << 27) // D))
        B = _log(rng, 1, min(8192, (1 << 25) // D))
        case = dict(kind=kind, V=V, D=D, B=B)
        if kind in ("embed_csr", "embed_mask"):
            return dict(case, density=round(rng.uniform(0.01, 0.5 if V * D < 1 << 25 else 0.1), 3))
        case["dtype"] = rng.choice(("f32", "f32", "bf16", "f16"))
        case["out"] = rng.choice(("f32", case["dtype"]))
        return dict(case, tied=rng.random() < 0.4) if kind == "embed_bwd" else case
    if kind.startswith("norm"):
        K = _log(rng, 10, 9216)
        B = _log(rng, 1, min(8192, 9216 * 2048 // K))
        return dict(kind=kind, K=K, B=B, dtype=rng.choice(("f32", "f32", "bf16", "f16")),
                    gate=rng.choice(("none", "row", "full")), sigmoid=rng.random() < 0.5, post=rng.random() < 0.7)
    layers, left = [], 100_000_000
    for _ in range(_log(rng, 1, 24)):
        n, k = _log(rng, 10, 4096), _log(rng, 10, 9216)
        if n * k > left:
            break
        left -= n * k
        layers += [f"{n}x{k}", f"{n}"]
    dtype = rng.choice(("f32", "f32", "bf16", "f16"))
    return dict(kind=kind, layers=",".join(layers), dtype=dtype, out=rng.choice(("f32", dtype)),
                grad_scale=rng.choice((1.0, 1024.0)), max_norm=rng.choice((1.0, 1.0, 1000.0)))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _tokens(case, g):
    V, B = case["V"], case["B"]
    u = torch.rand((B,), generator=g, device="cuda", dtype=torch.float64)
    t = ((u * math.log(V + 1)).exp().floor().long() - 1).clamp(0, V - 1).to(torch.int32)
    if B >= 16:
        t[B - B // 16:] = -1
    return t


def _sparse_table(case, g):
    """A CSR table whose rows hold from no entry to twice the average: the same number in all for every seed."""
    V, D = case["V"], case["D"]
    v = torch.arange(V, dtype=torch.float64)
    counts = (2 * case["density"] * D * ((v * 0.6180339887498949 + 0.5) % 1.0)).round().long().clamp_(0, D)
    counts[0] = counts[0].clamp_min(1)  # no table without an entry
    nnz, longest = int(counts.sum()), int(counts.max())
    row_ptr = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).cuda()
    rows = torch.repeat_interleave(torch.arange(V, device="cuda"), counts.cuda(), output_size=nnz)
    # entry j of n in a row: one of its columns j D / n .. (j + 1) D / n - 1
    j, n = torch.arange(nnz, device="cuda") - row_ptr[rows], counts.cuda()[rows]
    low, high = j * D // n, (j + 1) * D // n
    cols = low + (torch.rand((nnz,), generator=g, device="cuda", dtype=torch.float64) * (high - low)).long()
    vals = torch.randn((nnz,), generator=g, device="cuda") * 0.02
    return dict(row_ptr=row_ptr.to(torch.int32), col_idx=cols.to(torch.int32), vals=vals, nnz=nnz, longest=longest,
                rows=rows.to(torch.int32))


def _prepare_norm(case, g):
    K, B, T = case["K"], case["B"], TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    s = dict(alpha=1 / math.sqrt(2.0), gate=None, post=None)
    # features of very different size, as a residual stream has them
    sizes = (0.7 * normal(K, 1)).exp()
    r = (normal(K, B) * sizes).to(T)
    s["y"] = (normal(K, B) * (0.5 * normal(K, 1)).exp() * 0.3).to(T)
    s["pre"] = 1.0 + 0.2 * normal(K)
    if case["post"]:
        s["post"] = 0.5 + 0.2 * normal(K)
    if case["gate"] == "row":
        s["gate"] = 0.5 + 0.3 * normal(K)
    elif case["gate"] == "full":
        s["gate"] = (normal(K, B) + 0.5).to(T)
    if case["kind"] == "norm":
        s["r"] = r
        s["r_out"], s["h"] = torch.empty_like(r), torch.empty_like(r)
        return s
    s["r_out"] = _plain_norm(dict(s, r=r, case=case))["r"]
    s["dr_out"] = (normal(K, B) * 0.1).to(T)
    s["dh"] = (normal(K, B) * 0.1 * (0.5 * normal(K, 1)).exp()).to(T)
    return s


def _shapes(layers):
    return [tuple(int(n) for n in x.split("x")) for x in layers.split(",") if x]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    if kind.startswith("norm"):
        return dict(_prepare_norm(case, g), case=case)
    if kind == "clip":
        shapes, T = _shapes(case["layers"]), TYPES[case["dtype"]]
        total = sum(math.prod(x) for x in shapes)
        grads, out = [], []
        for shape in shapes:
            size = 5.0 / math.sqrt(total) * case["grad_scale"] * float(torch.rand((1,), generator=g, device="cuda") + 0.5)
            grads.append((torch.randn(shape, generator=g, device="cuda") * size).to(T))
            out.append(torch.empty(shape, dtype=TYPES[case["out"]], device="cuda"))
        return dict(case=case, grads=grads, out=out)
    V, D, B = case["V"], case["D"], case["B"]
    s = dict(case=case, tokens=_tokens(case, g), scale=math.sqrt(D))
    if kind in ("embed_csr", "embed_mask"):
        s.update(_sparse_table(case, g))
    if kind == "embed":
        s["E"] = (torch.randn((V, D), generator=g, device="cuda") * 0.02).to(TYPES[case["dtype"]])
    if kind in ("embed", "embed_csr"):
        s["X"] = torch.empty((D, B), device="cuda", dtype=TYPES[case.get("out", "f32")])
        return s
    s["dX"] = (torch.randn((D, B), generator=g, device="cuda") * 1e-2).to(TYPES[case.get("dtype", "f32")])
    if kind == "embed_mask":
        s["gv"] = torch.empty(s["nnz"], device="cuda")
        return s
    if case["tied"]:
        s["there"] = (torch.randn((V, D), generator=g, device="cuda") * 1e-2).to(TYPES[case["out"]])
    s["dE"] = torch.empty((V, D), device="cuda", dtype=TYPES[case["out"]])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_1905_07931_amd as L1
    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        return L1.embedding_fwd(s["E"], s["tokens"], X=s["X"], scale=s["scale"])
    if kind == "embed_csr":
        W = L1.CSR(case["V"], case["D"], s["row_ptr"], s["col_idx"], s["vals"], s["nnz"])
        return L1.embedding_fwd(W, s["tokens"], X=s["X"], scale=s["scale"])
    if kind == "embed_mask":
        W = L1.CSR(case["V"], case["D"], s["row_ptr"], s["col_idx"], s["vals"], s["nnz"])
        return L1.embedding_masked_bwd(W, s["dX"], s["tokens"], gv=s["gv"], scale=s["scale"])
    if kind == "embed_bwd":
        return L1.embedding_bwd(s["dX"], s["tokens"], case["V"], dE=s["dE"], scale=s["scale"], add=s.get("there"))
    if kind == "norm":
        r, h = L1.residual_norm_fwd(s["r"], s["y"], gate=s["gate"], post_gain=s["post"], pre_gain=s["pre"], alpha=s["alpha"],
                                    eps=EPS, sigmoid=case["sigmoid"], r_out=s["r_out"], h=s["h"])
        return {"r": r, "h": h}
    if kind == "norm_bwd":
        d = L1.residual_norm_bwd(s["r_out"], s["dr_out"], s["dh"], s["y"], gate=s["gate"], post_gain=s["post"],
                                 pre_gain=s["pre"], alpha=s["alpha"], eps=EPS, sigmoid=case["sigmoid"])
        out = {"dr": d.r, "dy": d.y, "dpre": d.pre_gain}
        if s["gate"] is not None:
            out["dgate"] = d.gate
        if s["post"] is not None:
            out["dpost"] = d.post_gain
        return out
    stats = L1.clip_grad_norm(s["grads"], case["max_norm"], grad_scale=case["grad_scale"], eps=EPS, out=s["out"])
    return {"stats": stats, "grads": s["out"]}


def _columns(rows, tokens, scale):
    """Rows of a table's lookup as columns, those of no token 0."""
    return (torch.where((tokens >= 0)[:, None], rows, torch.zeros_like(rows)) * scale).t().contiguous()


def _plain_table_gradient(s):
    V, tokens = s["case"]["V"], s["tokens"].long()
    rows = s["dX"].float().t() * s["scale"]
    rows = torch.where((tokens >= 0)[:, None], rows, torch.zeros_like(rows))
    return torch.zeros((V, s["case"]["D"]), device="cuda").index_add_(0, tokens.clamp_min(0), rows)


def _gate(s):
    """(a(gate), its derivative), as columns or whole; 1 without gate."""
    if s["gate"] is None:
        return 1.0, 0.0
    gate = s["gate"].float()
    if gate.dim() == 1:
        gate = gate[:, None]
    if not s["case"]["sigmoid"]:
        return gate, 1.0
    a = 1 / (1 + (-gate).exp())
    return a, a * (1 - a)


def _plain_norm(s):
    r, y, T = s["r"].float(), s["y"].float(), s["r"].dtype
    n = y
    if s["post"] is not None:
        n = y * ((y * y).mean(0) + EPS).rsqrt() * s["post"][:, None]
    r = r + s["alpha"] * _gate(s)[0] * n
    h = r * ((r * r).mean(0) + EPS).rsqrt() * s["pre"][:, None]
    return {"r": r.to(T), "h": h.to(T)}


def _plain_norm_bwd(s):
    r, y, dr, dh, T = s["r_out"].float(), s["y"].float(), s["dr_out"].float(), s["dh"].float(), s["r_out"].dtype
    a, da = _gate(s)
    inv = ((r * r).mean(0) + EPS).rsqrt()
    u = dh * s["pre"][:, None]
    t = dr + inv * u - inv ** 3 * (u * r).mean(0) * r
    out = {"dr": t.to(T), "dpre": (dh * r * inv).sum(1)}
    n = y
    if s["post"] is not None:
        q = (y * y).mean(0)
        q = (q + EPS).rsqrt()
        v = s["alpha"] * a * t
        out["dpost"] = (v * y * q).sum(1)
        n = y * q * s["post"][:, None]
        v = v * s["post"][:, None]
        out["dy"] = (q * v - q ** 3 * (v * y).mean(0) * y).to(T)
    else:
        out["dy"] = (s["alpha"] * a * t).to(T)
    if s["gate"] is not None:
        dg = s["alpha"] * t * n * da
        out["dgate"] = dg.sum(1) if s["gate"].dim() == 1 else dg.to(T)
    return out


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        rows = s["E"][s["tokens"].long().clamp_min(0)].float()
        return _columns(rows, s["tokens"], s["scale"]).to(TYPES[case["out"]])
    if kind == "embed_csr":
        D, B, t = case["D"], case["B"], s["tokens"].long().clamp_min(0)
        first, end = s["row_ptr"][t].long(), s["row_ptr"][t + 1].long()
        at = first[:, None] + torch.arange(s["longest"], device="cuda")
        inside = at < end[:, None]
        at = at.clamp_max(max(s["nnz"] - 1, 0))
        cols = torch.where(inside, s["col_idx"][at].long(), torch.full_like(at, D))  # what is past a row: column D, dropped
        rows = torch.zeros((B, D + 1), device="cuda").scatter_(1, cols, s["vals"][at])[:, :D]
        return _columns(rows, s["tokens"], s["scale"])
    if kind == "embed_mask":
        return _plain_table_gradient(s)[s["rows"].long(), s["col_idx"].long()]
    if kind == "embed_bwd":
        dE = _plain_table_gradient(s)
        if case["tied"]:
            dE += s["there"].float()
        return dE.to(TYPES[case["out"]])
    if kind == "norm":
        return _plain_norm(s)
    if kind == "norm_bwd":
        return _plain_norm_bwd(s)
    square = sum((x.float() * x.float()).sum() for x in s["grads"])
    norm = square.sqrt() / case["grad_scale"]
    factor = (case["max_norm"] / (norm + EPS)).clamp_max(1.0) / case["grad_scale"]
    T = TYPES[case["out"]]
    return {"stats": torch.stack([norm, factor]), "grads": [(x.float() * factor).to(T) for x in s["grads"]]}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it has to give
# ---------------------------------------------------------------------------

def _distinct(case):
    """Expected number of different tokens among those that are no padding."""
    V, B = case["V"], case["B"]
    n = B - B // 16 if B >= 16 else B
    v = torch.arange(V, dtype=torch.float64)
    return float((1 - (1 - ((v + 2) / (v + 1)).log() / math.log(V + 1)) ** n).sum())


def work(case):
    kind = case["kind"]
    if kind == "clip":
        n = sum(math.prod(x) for x in _shapes(case["layers"]))
        return {"bytes": n * (BYTES[case["dtype"]] + BYTES[case["out"]]), "flops": 3 * n}
    if kind.startswith("norm"):
        n, e = case["K"] * case["B"], BYTES[case["dtype"]]
        full = case["gate"] == "full"
        if kind == "norm":
            return {"bytes": n * e * (4 + full) + 8 * case["K"], "flops": 14 * n}
        return {"bytes": n * e * (6 + 2 * full) + 16 * case["K"], "flops": 30 * n}
    V, D, B = case["V"], case["D"], case["B"]
    rows = _distinct(case)
    if kind == "embed":
        return {"bytes": rows * D * BYTES[case["dtype"]] + D * B * BYTES[case["out"]] + 4 * B, "flops": D * B}
    if kind == "embed_csr":
        return {"bytes": rows * D * case["density"] * 8 + 4 * D * B + 4 * B, "flops": D * B * case["density"]}
    if kind == "embed_mask":
        n = V * D * case["density"]  # the pattern's columns are needed where a row has tokens
        return {"bytes": 4 * D * B + 4 * n + 4 * n * rows / V + 4 * V, "flops": 2 * D * B * case["density"]}
    out = BYTES[case["out"]]
    return {"bytes": D * B * BYTES[case["dtype"]] + V * D * out * (1 + case["tied"]) + 4 * B, "flops": 2 * D * B}


def _exact_norm(r, y, gate, post, pre, case, alpha):
    """r' and h in 64 bits."""
    n = y
    if post is not None:
        n = y / (y.square().mean(0, keepdim=True) + EPS).sqrt() * post.unsqueeze(1)
    if gate is not None:
        gate = gate.unsqueeze(1) if gate.dim() == 1 else gate
        n = n * (torch.sigmoid(gate) if case["sigmoid"] else gate)
    r = torch.add(r, n, alpha=alpha)
    return r, r / (r.square().mean(0, keepdim=True) + EPS).sqrt() * pre.unsqueeze(1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if kind == "clip":
        norm = math.sqrt(sum(float(x.double().norm() ** 2) for x in s["grads"])) / case["grad_scale"]
        factor = min(1.0, case["max_norm"] / (norm + EPS)) / case["grad_scale"]
        return {"stats": torch.tensor([norm, factor], dtype=torch.float64, device="cuda"),
                "grads": [x.double() * factor for x in s["grads"]]}
    if kind == "norm":
        r, h = _exact_norm(wide["r"], wide["y"], wide.get("gate"), wide.get("post"), wide["pre"], case, s["alpha"])
        return {"r": r, "h": h}
    if kind == "norm_bwd":
        # the gradients of the forward definition, r' being given: h as a function of r', r' as one of y, the gate, the gain
        named = {k: wide[k].requires_grad_() for k in ("r_out", "pre", "y", "gate", "post") if k in wide}
        zero = torch.zeros_like(wide["r_out"])
        moved, _ = _exact_norm(zero, named["y"], named.get("gate"), named.get("post"), wide["pre"].detach(), case, s["alpha"])
        r = named["r_out"]
        h = r / (r.square().mean(0, keepdim=True) + EPS).sqrt() * named["pre"].unsqueeze(1)
        through, dpre = torch.autograd.grad(h, (r, named["pre"]), wide["dh"])
        t = wide["dr_out"] + through
        rest = [k for k in ("y", "gate", "post") if k in named]
        grads = dict(zip(rest, torch.autograd.grad(moved, [named[k] for k in rest], t)))
        return {"dr": t, "dpre": dpre, **{"d" + k: v for k, v in grads.items()}}
    V, D, B = case["V"], case["D"], case["B"]
    tokens = s["tokens"].long()
    good = (tokens >= 0).nonzero().squeeze(1)
    if kind in ("embed", "embed_csr"):
        table = wide.get("E")
        if table is None:
            table = torch.sparse_csr_tensor(s["row_ptr"].long(), s["col_idx"].long(), wide["vals"], (V, D)).to_dense()
        X = torch.zeros((D, B), dtype=torch.float64, device="cuda")
        X[:, good] = table.index_select(0, tokens[good]).mul_(s["scale"]).t()
        return X
    # by sorted tokens: differences of running sums would lose bits, so segment by segment through a sum over equal tokens
    values, of = tokens[good].unique(return_inverse=True)
    rows = torch.zeros((values.numel(), D), dtype=torch.float64, device="cuda")
    rows.index_add_(0, of, wide["dX"].t().contiguous().index_select(0, good))
    rows *= s["scale"]
    if kind == "embed_mask":
        where = torch.full((V,), -1, dtype=torch.int64, device="cuda")
        where[values] = torch.arange(values.numel(), device="cuda")
        row = where[s["rows"].long()]
        got = rows[row.clamp_min(0), s["col_idx"].long()] if values.numel() else torch.zeros(s["nnz"], device="cuda").double()
        return torch.where(row >= 0, got, torch.zeros_like(got))
    dE = wide["there"] if case["tied"] else torch.zeros((V, D), dtype=torch.float64, device="cuda")
    return dE.index_add_(0, values, rows)
