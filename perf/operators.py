"""Cases of the small-batch and optimiser operators of the MoE FFN layer, each with a plain form.

Three operators, on the weights of one layer:

* ``few``    ``moevie_moe_few``: the whole layer (router, selection, gates, experts, shared
             expert, combine) for 1 to 64 tokens, as an interactive or token-by-token caller
             needs it;
* ``ortho``  ``moevie_orthogonalize``: every matrix of a stack replaced by the Newton-Schulz
             approximation of its orthogonal factor;
* ``muon``   ``moevie_muon_update``: one optimiser step on a stack of expert matrices (momentum,
             orthogonalised update, weight decay, fp32 master weights and their bf16 copy).

``run`` computes a case with the library where ``own`` is true and with elementary torch
operations in 32 bits otherwise.
"""
import math

import torch

own = False

STEPS = 5
COEF = (3.4445, -4.7750, 2.0315)   # X <- a X + (b A + c A^2) X, A = X X^T


def listed():
    few = {"op": "few", "hs": 0, "act": "gelu", "skew": 0.0}
    return [
        # one token through the smallest layer: latency alone
        {"name": "few-1-small", **few, "T": 1, "d": 768, "E": 16, "k": 2, "h": 768},
        # one token through a batch-1 image layer: eight experts' weights are read once
        {"name": "few-1", **few, "T": 1, "d": 1536, "E": 64, "k": 8, "h": 768},
        # a handful of tokens, SwiGLU experts of an odd width and a shared expert
        {"name": "few-5-swiglu", **few, "T": 5, "d": 1280, "E": 31, "k": 7, "h": 854, "hs": 854, "act": "swiglu"},
        # sixteen tokens, skewed loads: some experts see most tokens, many none
        {"name": "few-16-skew", **few, "T": 16, "d": 1536, "E": 128, "k": 8, "h": 384, "skew": 1.0},
        # 64 tokens, a shared expert that every token visits
        {"name": "few-64-shared", **few, "T": 64, "d": 1024, "E": 64, "k": 8, "h": 512, "hs": 1024},
        # 64 tokens over many narrow experts: nearly every expert is read
        {"name": "few-64-wide", **few, "T": 64, "d": 1664, "E": 256, "k": 8, "h": 416},
        # one square matrix (a shared expert's): the chain of products is all latency
        {"name": "ortho-1", "op": "ortho", "N": 1, "r": 1024, "c": 1024, "dtype": "f32", "rank": 0},
        # sixteen square matrices from a 16-bit update
        {"name": "ortho-16-b16", "op": "ortho", "N": 16, "r": 768, "c": 768, "dtype": "bf16", "rank": 0},
        # the down-projections of 256 narrow experts: wide matrices
        {"name": "ortho-256", "op": "ortho", "N": 256, "r": 416, "c": 1664, "dtype": "f32", "rank": 0},
        # a step on tall matrices, gradients from a few hundred tokens for each expert
        {"name": "muon-64", "op": "muon", "N": 64, "r": 1024, "c": 512, "rank": 256, "nesterov": True},
        # odd widths, gradients of few tokens
        {"name": "muon-31-odd", "op": "muon", "N": 31, "r": 1280, "c": 854, "rank": 64, "nesterov": True},
        # the up-projections of 256 narrow experts
        {"name": "muon-256", "op": "muon", "N": 256, "r": 1664, "c": 416, "rank": 0, "nesterov": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["few", "few", "ortho", "muon"])
    if op == "few":
        act = rng.choice(["gelu", "swiglu"])
        T, d, h, E = _log(rng, 1, 64), 8 * _log(rng, 32, 256), _log(rng, 64, 1024), _log(rng, 8, 256)
        E = max(8, min(E, 350_000_000 // (d * h * (3 if act == "swiglu" else 2))))
        k = rng.randint(1, 8)
        hs = rng.choice([0, 0, h, _log(rng, 64, 1024)])
        return {"op": op, "T": T, "d": d, "E": E, "k": k, "h": h, "hs": hs, "act": act, "skew": rng.choice([0.0, 1.0])}
    r, c = _log(rng, 64, 2048), _log(rng, 64, 2048)
    m, n = min(r, c), max(r, c)
    most = min(150_000_000 // (r * c), int(1.0e12 / (STEPS * (3 * m * m * n + m ** 3))))
    N = _log(rng, 1, max(1, min(256, most)))
    rank = rng.choice([0, max(1, m // rng.randint(2, 8))])
    if op == "ortho":
        return {"op": op, "N": N, "r": r, "c": c, "dtype": rng.choice(["f32", "bf16"]), "rank": rank}
    return {"op": op, "N": N, "r": r, "c": c, "rank": rank, "nesterov": rng.choice([True, False])}


# ------------------------------------------------------------------ inputs

def _ld(h):
    return (h + 7) // 8 * 8


def _rows(shape, dtype, fill):
    """A tensor [..., h] whose rows start 16 bytes apart (as the library takes W1 and its like)."""
    buf = torch.zeros(*shape[:-1], _ld(shape[-1]), dtype=dtype, device="cuda")
    v = buf[..., :shape[-1]]
    v.copy_(fill)
    return v


def _few_inputs(case, g):
    T, d, E, k, h, hs = (case[n] for n in ("T", "d", "E", "k", "h", "hs"))

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    s = {"W_r": normal(d, E, std=0.02), "b": torch.rand(E, generator=g, device="cuda") * 0.2 - 0.1}
    if case["skew"]:   # a constant feature carries each expert's popularity
        order = torch.randperm(E, generator=g, device="cuda")
        s["W_r"][d - 1] = -case["skew"] * torch.log1p(order.float())
    spare = T + max(8, T // 4)
    x = normal(spare, d).to(torch.bfloat16)
    if case["skew"]:
        x[:, d - 1] = 1.0
    # Keep tokens whose k-th and (k+1)-th keys are further apart than 32-bit logits can blur:
    # nearer ones (one token in some thousands) have no answer that a 32-bit form must give.
    key = torch.sigmoid(x.double() @ s["W_r"].double()) + s["b"].double()
    top = torch.sort(key, dim=1, descending=True)[0]
    near = (top[:, k - 1] - top[:, k] < 2e-5) if k < E else torch.zeros(spare, dtype=torch.bool, device="cuda")
    s["x"] = x[torch.sort(near.int(), stable=True)[1][:T]].contiguous()
    s["W1"] = _rows((E, d, h), torch.bfloat16, normal(E, d, h, std=d ** -0.5))
    s["W2"] = normal(E, h, d, std=h ** -0.5).to(torch.bfloat16)
    swiglu = case["act"] == "swiglu"
    s["W3"] = _rows((E, d, h), torch.bfloat16, normal(E, d, h, std=d ** -0.5)) if swiglu else None
    s["Ws1"] = s["Ws2"] = s["Ws3"] = None
    if hs:
        s["Ws1"] = _rows((d, hs), torch.bfloat16, normal(d, hs, std=d ** -0.5))
        s["Ws2"] = normal(hs, d, std=hs ** -0.5).to(torch.bfloat16)
        s["Ws3"] = _rows((d, hs), torch.bfloat16, normal(d, hs, std=d ** -0.5)) if swiglu else None
    return s


def _gradients(N, r, c, rank, g):
    """Gradients of expert matrices: sums of `rank` outer products (one for each token that the
    expert saw) on a scale of their own for each expert, or full-rank noise for rank 0."""
    scale = torch.exp(2 * torch.randn(N, 1, 1, generator=g, device="cuda")) * 1e-3
    if not rank:
        return torch.randn(N, r, c, generator=g, device="cuda") * scale
    a = torch.randn(N, r, rank, generator=g, device="cuda")
    b = torch.randn(N, rank, c, generator=g, device="cuda")
    return torch.bmm(a, b) * scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    if case["op"] == "few":
        s = _few_inputs(case, g)
    elif case["op"] == "ortho":
        u = _gradients(case["N"], case["r"], case["c"], case["rank"], g)
        s = {"U": u.to(torch.bfloat16) if case["dtype"] == "bf16" else u}
    else:
        N, r, c = case["N"], case["r"], case["c"]
        w = torch.randn(N, r, c, generator=g, device="cuda") * r ** -0.5
        s = {"W": _rows((N, r, c), torch.float32, w), "Wb": _rows((N, r, c), torch.bfloat16, w)}
        s["M"] = _rows((N, r, c), torch.float32, _gradients(N, r, c, 0, g))
        s["G"] = _rows((N, r, c), torch.float32, _gradients(N, r, c, case["rank"], g))
        # a fine-tuning step
        s.update(lr=5e-5, momentum=0.95, weight_decay=0.1, scale=0.2 * math.sqrt(max(r, c)))
    s["case"] = case
    if own:   # what a program keeps beside its weights: the workspace
        from paper_2608_17402_gb300 import moevie
        if case["op"] == "few":
            s["layer"] = moevie.LayerWeights(W_r=s["W_r"], b=s["b"], W1=s["W1"], W2=s["W2"], k=case["k"],
                                             Ws1=s["Ws1"], Ws2=s["Ws2"], lam=1.0, W3=s["W3"], Ws3=s["Ws3"])
            s["ws"] = moevie.FewWorkspace(case["T"], case["d"], case["E"], case["k"], case["h"], case["hs"])
        else:
            s["ws"] = moevie.OrthoWorkspace(case["N"], case["r"], case["c"])
    return s


# -------------------------------------------------------------- plain forms

def _act(u, v):
    if v is None:
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    return u / (1 + torch.exp(-u)) * v


def _few_plain(s):
    k = s["case"]["k"]
    x = s["x"].float()
    T, d = x.shape
    sig = 1 / (1 + torch.exp(-(x @ s["W_r"])))
    order = torch.sort(sig + s["b"], dim=1, descending=True, stable=True)[1]
    idx = torch.sort(order[:, :k], dim=1)[0]
    gate = torch.gather(sig, 1, idx)
    gate = gate / gate.sum(1, keepdim=True)
    e = idx.reshape(-1)
    xs = x.repeat_interleave(k, 0).unsqueeze(1)                       # [T k, 1, d]
    u = torch.bmm(xs, s["W1"][e].float())
    v = torch.bmm(xs, s["W3"][e].float()) if s["W3"] is not None else None
    rows = torch.bmm(_act(u, v), s["W2"][e].float()).view(T, k, d)
    y = (gate.unsqueeze(2) * rows).sum(1)
    if s["Ws1"] is not None:
        v = x @ s["Ws3"].float() if s["Ws3"] is not None else None
        y = y + _act(x @ s["Ws1"].float(), v) @ s["Ws2"].float()
    return {"y": y.to(torch.bfloat16), "idx": idx.to(torch.int32), "gate": gate}


def _newton_schulz_plain(u):
    x = u.float()
    if x.shape[1] > x.shape[2]:
        return _newton_schulz_plain(x.transpose(1, 2)).transpose(1, 2)
    norm = torch.sqrt((x * x).sum((1, 2), keepdim=True))
    x = torch.where(norm > 0, x / norm, torch.zeros_like(x))
    a, b, c = COEF
    for _ in range(STEPS):
        g = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * g + c * torch.bmm(g, g), x)
    return x


def _muon_plain(s):
    s["M"].mul_(s["momentum"]).add_(s["G"])
    u = s["G"] + s["momentum"] * s["M"] if s["case"]["nesterov"] else s["M"]
    o = _newton_schulz_plain(u)
    s["W"].mul_(1 - s["lr"] * s["weight_decay"]).sub_(o, alpha=s["lr"] * s["scale"])
    s["Wb"].copy_(s["W"])
    return {"W": s["W"], "Wb": s["Wb"], "M": s["M"]}


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "few":
            return _few_plain(s)
        if op == "ortho":
            return {"O": _newton_schulz_plain(s["U"]).to(torch.bfloat16)}
        return _muon_plain(s)
    from paper_2608_17402_gb300 import moevie
    if op == "few":
        y, idx, gate = moevie.moevie_moe_few(s["layer"], s["x"], s["ws"], routing=True)
        return {"y": y, "idx": idx, "gate": gate}
    if op == "ortho":
        return {"O": moevie.moevie_orthogonalize(s["U"], s["ws"], coef=COEF, steps=STEPS)}
    moevie.moevie_muon_update(s["W"], s["M"], s["G"], s["ws"], lr=s["lr"], momentum=s["momentum"],
                              weight_decay=s["weight_decay"], nesterov=s["case"]["nesterov"], scale=s["scale"],
                              W_bf16=s["Wb"], coef=COEF, steps=STEPS)
    return {"W": s["W"], "Wb": s["Wb"], "M": s["M"]}


# ------------------------------------------------------------ work, 64 bits

def work(case):
    if case["op"] == "few":
        T, d, E, k, h, hs = (case[n] for n in ("T", "d", "E", "k", "h", "hs"))
        mats = 3 if case["act"] == "swiglu" else 2
        touched = E * (1 - (1 - k / E) ** T)   # expected number of experts that some token selects
        nbytes = mats * 2 * d * (touched * h + hs) + 4 * d * E + 4 * E + 4 * T * d + 8 * T * k
        return {"bytes": nbytes, "flops": 2 * T * d * (mats * (k * h + hs) + E)}
    N, r, c = case["N"], case["r"], case["c"]
    m, n = min(r, c), max(r, c)
    # X X^T and A A^T are symmetric: half of each product is the other half mirrored
    flops = N * STEPS * (3.0 * m * m * n + 1.0 * m * m * m)
    if case["op"] == "ortho":
        return {"bytes": N * r * c * ((2 if case["dtype"] == "bf16" else 4) + 2), "flops": flops}
    return {"bytes": N * r * c * (4 + 8 + 8 + 2), "flops": flops}   # G, M twice, W twice, the bf16 copy


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "few":
        x = s["x"].to(f64)
        sig = torch.special.expit(torch.einsum("td,de->te", x, s["W_r"].to(f64)))
        key = (sig + s["b"].to(f64)).cpu()
        ids = [sorted(sorted(range(case["E"]), key=lambda e: (-row[e], e))[:case["k"]]) for row in key.tolist()]
        idx = torch.tensor(ids, dtype=torch.int64, device="cuda")
        gate = sig.gather(1, idx)
        gate /= gate.sum(dim=1, keepdim=True)

        def ffn(z, w1, w3, w2):
            u = z @ w1.to(f64)
            if w3 is None:
                a = u * torch.special.ndtr(u)
            else:
                a = u * torch.special.expit(u) * (z @ w3.to(f64))
            return a @ w2.to(f64)

        y = torch.zeros_like(x)
        for e in sorted({e for row in ids for e in row}):
            t, j = (idx == e).nonzero(as_tuple=True)
            w3 = s["W3"][e] if s["W3"] is not None else None
            y[t] += gate[t, j, None] * ffn(x[t], s["W1"][e], w3, s["W2"][e])
        if s["Ws1"] is not None:
            y += ffn(x, s["Ws1"], s["Ws3"], s["Ws2"])
        return {"y": y, "idx": idx.to(torch.int32), "gate": gate}

    def orthogonal(u):   # one matrix
        z = u.to(f64)
        norm = torch.linalg.matrix_norm(z)
        if norm == 0:
            return z
        z = z / norm
        flip = z.shape[0] > z.shape[1]
        z = z.mT if flip else z
        eye = torch.eye(z.shape[0], dtype=f64, device=z.device)
        for _ in range(STEPS):
            gram = z @ z.mT
            z = (COEF[0] * eye + gram @ (COEF[1] * eye + COEF[2] * gram)) @ z
        return z.mT if flip else z

    if case["op"] == "ortho":
        return {"O": torch.stack([orthogonal(u) for u in s["U"]])}
    G, W, mu = s["G"].to(f64), s["W"].to(f64), s["momentum"]
    M = mu * s["M"].to(f64) + G
    U = G + mu * M if case["nesterov"] else M
    O = torch.stack([orthogonal(u) for u in U])
    W = W - s["lr"] * (s["weight_decay"] * W + s["scale"] * O)
    return {"W": W, "Wb": W.clone(), "M": M}
