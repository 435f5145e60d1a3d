"""Cases of the operators of a training step around the MoE FFN layer, each with a plain form.

Three operators, on the rows that a block of the encoder keeps and passes on:

* ``join``     ``moevie_residual_norm``: the layer's output normed, gated and added to the scaled
               residual stream, and the norm before the next layer, in one pass; with ``save`` also
               the 8-bit checkpoints of what it read.  ``join-bwd`` is its backward,
               ``moevie_residual_norm_backward``, from rows kept whole or in 8 bits;
* ``balance``  ``moevie_balance_loss``: the auxiliary loss of expert loads, the loads themselves
               and the gradient of the router's logits;
* ``keep``     ``moevie_checkpoint_store`` and ``moevie_checkpoint_load``: activations kept in 8 bits
               after the forward and read back for the backward.

``run`` computes a case with the library where ``own`` is true and with elementary torch
operations in 32 bits otherwise.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128   # columns that share a scale in a checkpoint


def listed():
    join = {"res": "bf16", "pre": "rms", "post": "rms", "bias": False, "gate": True, "G": 1, "alpha": 1.0}
    image = {"res": "bf16", "pre": "layer", "post": "layer", "bias": True, "gate": True, "G": 1, "alpha": 1.0}
    deep = {"res": "f32", "pre": "layer", "post": "rms", "bias": True, "gate": True, "alpha": 0.75}
    return [
        # one token of a decoding step: latency alone
        {"name": "join-1", "op": "join", "T": 1, "d": 768, "save": False, **join},
        # 32 images of 256 patches, a step that keeps 8-bit checkpoints
        {"name": "join-images-save", "op": "join", "T": 8192, "d": 1024, "save": True, **image},
        # the largest batch, residual stream in 32 bits, a gate for each of 63 ragged clips
        {"name": "join-clips-f32", "op": "join", "T": 65536, "d": 1664, "save": False, "G": 63, **deep},
        # one small image: the gradients of the weights are most of the work after the rows
        {"name": "join-bwd-image", "op": "join-bwd", "T": 257, "d": 768, "saved": "whole", "du": "bf16", **image},
        # 32 images, everything read back from 8-bit checkpoints
        {"name": "join-bwd-images-q8", "op": "join-bwd", "T": 8192, "d": 1280, "saved": "q8", "du": "f32", **join},
        # the largest batch, 32-bit residual stream and gradients, ragged clips
        {"name": "join-bwd-clips-f32", "op": "join-bwd", "T": 65536, "d": 1664, "saved": "whole", "du": "f32", "G": 63,
         **deep},
        # two images through the smallest router: latency
        {"name": "balance-small", "op": "balance", "T": 512, "E": 16, "k": 2, "score": "softmax", "G": 1, "skew": 0.0},
        # 32 images, each balanced by itself, the layer's sigmoid scores, an odd number of experts
        {"name": "balance-images", "op": "balance", "T": 8192, "E": 31, "k": 7, "score": "sigmoid", "G": 32, "skew": 0.5},
        # the largest batch and router, one balance over all tokens, skewed loads
        {"name": "balance-batch", "op": "balance", "T": 65536, "E": 256, "k": 8, "score": "sigmoid", "G": 1, "skew": 1.0},
        # one small image, an odd number of tokens, a width that leaves a part of a block
        {"name": "keep-image", "op": "keep", "T": 197, "d": 1288, "res": "bf16"},
        # a batch of clips, the layer's input kept for its backward
        {"name": "keep-clips", "op": "keep", "T": 32768, "d": 1536, "res": "bf16"},
        # the largest batch's residual stream, 32 bits before and after
        {"name": "keep-batch-f32", "op": "keep", "T": 65536, "d": 1664, "res": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["join", "join-bwd", "balance", "join", "join-bwd", "balance", "keep"])
    if op == "balance":
        E = _log(rng, 4, 1024)
        T = _log(rng, 1, min(65536, 65536 * 256 // E))
        return {"op": op, "T": T, "E": E, "k": rng.randint(1, min(8, E // 2)), "score": rng.choice(["softmax", "sigmoid"]),
                "G": rng.choice([1, _log(rng, 1, max(1, min(T, 256)))]), "skew": rng.choice([0.0, 1.0])}
    d = 8 * _log(rng, 8, 1024)
    T = _log(rng, 1, min(65536, 65536 * 1664 // d))
    if op == "keep":
        return {"op": op, "T": T, "d": d, "res": rng.choice(["bf16", "f32"])}
    case = {"op": op, "T": T, "d": d, "res": rng.choice(["bf16", "f32"]), "pre": rng.choice(["rms", "layer"]),
            "post": rng.choice(["rms", "layer", "none"]), "bias": rng.choice([False, True]),
            "gate": rng.choice([True, True, False]), "alpha": rng.choice([1.0, 0.75])}
    case["G"] = rng.choice([1, _log(rng, 1, max(1, min(T, 256)))]) if case["gate"] else 1
    if op == "join":
        return {**case, "save": rng.choice([False, True])}
    return {**case, "saved": rng.choice(["whole", "q8"]), "du": rng.choice(["f32", "bf16"])}


# ------------------------------------------------------------------ inputs

def _segments(T, G, g):
    """Ends of G runs of tokens, ragged, none longer than about three times the mean."""
    w = torch.rand(G, generator=g, device="cuda") + 0.25
    ends = torch.round(torch.cumsum(w, 0) / w.sum() * T).to(torch.int32)
    ends[-1] = T
    return torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), ends])


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _quantise(x):
    """Codes and scales of the 8-bit checkpoint of rows x [T, d]: the whole number nearest to 127 x / amax
    (an even one between two), decided in 64 bits, and amax / 127."""
    T, d = x.shape
    nb = -(-d // BLOCK)
    v = torch.zeros(T, nb * BLOCK, device="cuda")
    v[:, :d] = x
    v = v.view(T, nb, BLOCK)
    amax = v.abs().amax(2)
    some = amax >= 2.0 ** -110
    code = torch.round(torch.where(some[:, :, None], 127 * v.double() / amax.double()[:, :, None], 0.0)).to(torch.int8)
    return code.view(T, nb * BLOCK)[:, :d].contiguous(), torch.where(some, amax / 127.0, torch.zeros_like(amax))


def _values(code, scale):
    """What a checkpoint stands for, in 32 bits."""
    return code.float() * scale.repeat_interleave(BLOCK, 1)[:, :code.shape[1]]


def _stats(x, kind, eps=EPS):
    """(mean, 1 / deviation) of every row, [T, 2]; the mean is 0 for an RMS norm."""
    x = x.double()
    mean = x.mean(1) if kind == "layer" else torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
    rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return torch.stack([mean, rstd], 1).float()


def _join_inputs(case, g):
    T, d, G = case["T"], case["d"], case["G"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    s = {"seg": _segments(T, G, g) if G > 1 else None}
    post = case["post"] != "none"
    s["w_pre"], s["w_post"] = 1 + normal(d, std=0.2), 1 + normal(d, std=0.2) if post else None
    s["b_pre"], s["b_post"] = normal(d, std=0.1), normal(d, std=0.1) if post else None
    if not case["bias"]:
        s["b_pre"] = s["b_post"] = None
    s["gate"] = 0.1 + normal(G, d, std=0.1) if case["gate"] else None
    # a residual stream: channels of very different sizes, a common offset
    channel = torch.exp(normal(d, std=0.7))
    s["r"] = (normal(T, d) * channel + 0.1).to(_dtype(case["res"]))
    s["f"] = (normal(T, d) * torch.exp(normal(T, 1, std=0.5))).to(torch.bfloat16)
    if case["op"] == "join-bwd":
        s["stats_pre"] = _stats(s["r"], case["pre"])
        s["stats_post"] = _stats(s["f"], case["post"]) if case["post"] != "none" else None
        s["dr"] = normal(T, d, std=1e-3).to(_dtype(case["res"]))
        s["du"] = normal(T, d, std=1e-3).to(_dtype(case["du"]))
        if case["saved"] == "q8":   # what the forward left: codes and scales in place of the rows
            s["r"], s["f"] = _quantise(s["r"].float()), _quantise(s["f"].float())
    return s


def _balance_inputs(case, g):
    T, E, k = case["T"], case["E"], case["k"]
    s = {"seg": _segments(T, case["G"], g) if case["G"] > 1 else None}
    logits = torch.randn(T, E, generator=g, device="cuda")
    if case["skew"]:
        order = torch.randperm(E, generator=g, device="cuda")
        logits -= case["skew"] * torch.log1p(order.float())
    s["s"] = logits
    s["idx"] = torch.sort(torch.topk(logits, k, dim=1)[1], dim=1)[0].to(torch.int32)
    s["coef"] = 0.01
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op = case["op"]
    if op in ("join", "join-bwd"):
        s = _join_inputs(case, g)
    elif op == "balance":
        s = _balance_inputs(case, g)
    else:
        x = torch.randn(case["T"], case["d"], generator=g, device="cuda")
        x *= torch.exp(0.7 * torch.randn(case["d"], generator=g, device="cuda"))
        s = {"x": x.to(_dtype(case["res"]))}
    s["case"] = case
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """What a training program keeps beside its weights: the description of the block's norms, the
    workspace, and the buffers that every step writes anew."""
    from paper_2608_17402_gb300 import moevie
    case = s["case"]
    T, op = case["T"], case["op"]
    if op == "balance":
        s["ws"] = moevie.BalanceWorkspace(T, case["E"], case["k"], case["G"])
        s["out"] = moevie.BalanceOut.empty(T, case["E"], case["G"])
        return
    d, res = case["d"], _dtype(case["res"])
    if op == "keep":
        s["ck"], s["out"] = moevie.Checkpoint.empty(T, d), torch.empty_like(s["x"])
        return
    s["norms"] = moevie.ResidualNorm(d, pre=case["pre"], post=None if case["post"] == "none" else case["post"],
                                     w_pre=s["w_pre"], b_pre=s["b_pre"], w_post=s["w_post"], b_post=s["b_post"],
                                     gate=s["gate"], seg=s["seg"], residual_scale=case["alpha"], eps=EPS)
    s["ws"] = moevie.ResidualNormWorkspace(T, d, case["G"])
    if op == "join":
        s["out"] = moevie.ResidualNormOut.empty(s["norms"], T, res, save=case["save"])
        s["kept_r"], s["kept_f"] = (torch.empty_like(s[n]) if case["save"] else None for n in ("r", "f"))
    else:
        s["out"] = moevie.ResidualNormGrads.empty(s["norms"], T, res)
        if case["saved"] == "q8":
            s["r"], s["f"] = moevie.Checkpoint(*s["r"]), moevie.Checkpoint(*s["f"])


# -------------------------------------------------------------- plain forms

def _groups(seg, T):
    """The run that every token belongs to."""
    G = seg.numel() - 1
    return torch.repeat_interleave(torch.arange(G, device="cuda"), (seg[1:] - seg[:-1]).long(), output_size=T)


def _norm(x, kind, w, b):
    if kind == "none":
        return x, None
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros(x.shape[0], 1, device="cuda")
    z = x - mean
    rstd = 1 / torch.sqrt((z * z).mean(1, keepdim=True) + EPS)
    y = z * rstd * w
    return (y + b if b is not None else y), torch.cat([mean, rstd], 1)


def _gate_rows(s):
    gate = s["gate"]
    return gate if gate is None or s["seg"] is None else gate[_groups(s["seg"], s["case"]["T"])]


def _join_plain(s):
    case = s["case"]
    n, stats_post = _norm(s["f"].float(), case["post"], s["w_post"], s["b_post"])
    gate = _gate_rows(s)
    r1 = case["alpha"] * s["r"].float() + (n if gate is None else gate * n)
    u, stats_pre = _norm(r1, case["pre"], s["w_pre"], s["b_pre"])
    out = {"r": r1.to(s["r"].dtype), "u": u.to(torch.bfloat16), "stats_pre": stats_pre, "stats_post": stats_post}
    if case["save"]:
        out["kept_r"] = _values(*_quantise(s["r"].float())).to(s["r"].dtype)
        out["kept_f"] = _values(*_quantise(s["f"].float())).to(torch.bfloat16)
    return out


def _norm_back(g, xhat, rstd, kind):
    g = g - xhat * (g * xhat).mean(1, keepdim=True) - (g.mean(1, keepdim=True) if kind == "layer" else 0.0)
    return g * rstd


def _join_back_plain(s):
    case = s["case"]
    G, T, d = case["G"], case["T"], case["d"]
    r = _values(*s["r"]) if case["saved"] == "q8" else s["r"].float()
    f = _values(*s["f"]) if case["saved"] == "q8" else s["f"].float()
    du = s["du"].float()
    mean, rstd = s["stats_pre"][:, :1], s["stats_pre"][:, 1:]
    x1 = (r - mean) * rstd
    total = s["dr"].float() + _norm_back(du * s["w_pre"], x1, rstd, case["pre"])
    out = {"dr": (case["alpha"] * total).to(s["dr"].dtype), "dw_pre": (du * x1).sum(0)}
    out["db_pre"] = du.sum(0) if s["b_pre"] is not None else None
    gate = _gate_rows(s)
    gated = total if gate is None else gate * total
    out["dw_post"] = out["db_post"] = out["dgate"] = None
    n = f
    if case["post"] == "none":
        df = gated
    else:
        mean, rstd = s["stats_post"][:, :1], s["stats_post"][:, 1:]
        x2 = (f - mean) * rstd
        df = _norm_back(gated * s["w_post"], x2, rstd, case["post"])
        out["dw_post"] = (gated * x2).sum(0)
        n = x2 * s["w_post"]
        if s["b_post"] is not None:
            out["db_post"] = gated.sum(0)
            n = n + s["b_post"]
    out["df"] = df.to(torch.bfloat16)
    if gate is not None:
        if s["seg"] is None:
            out["dgate"] = (total * n).sum(0, keepdim=True)
        else:
            out["dgate"] = torch.zeros(G, d, device="cuda").index_add_(0, _groups(s["seg"], T), total * n)
    return out


def _balance_plain(s):
    case = s["case"]
    T, E, k, G = (case[n] for n in ("T", "E", "k", "G"))
    logits = s["s"]
    if s["seg"] is None:
        group, lengths = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.full((1, 1), T, device="cuda")
    else:
        group, lengths = _groups(s["seg"], T), (s["seg"][1:] - s["seg"][:-1]).unsqueeze(1)
    flat = (group[:, None] * E + s["idx"]).reshape(-1)
    counts = torch.zeros(G * E, dtype=torch.int32, device="cuda")
    counts.index_add_(0, flat, torch.ones_like(flat, dtype=torch.int32))
    counts = counts.view(G, E)
    # loads less the even load k / E: the probabilities add up to 1, so that this moves the loss by
    # coef alone, and nothing is lost where the loads are nearly even
    c = (s["coef"] * E / (k * T)) * (counts.double() / torch.clamp(lengths, min=1) - k / E)
    c = torch.where(counts * E == k * lengths, 0.0, c).float()
    if case["score"] == "softmax":
        p = torch.exp(logits - logits.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
        slope = p
    else:
        sig = 1 / (1 + torch.exp(-logits))
        p = sig / sig.sum(1, keepdim=True)
        slope = p * (1 - sig)
    c = c[group]
    dot = (p * c).sum(1, keepdim=True)
    return {"loss": s["coef"] + dot.sum().reshape(1), "counts": counts, "ds": slope * (c - dot)}


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "join":
            return _join_plain(s)
        if op == "join-bwd":
            return _join_back_plain(s)
        if op == "balance":
            return _balance_plain(s)
        return {"x": _values(*_quantise(s["x"].float())).to(s["x"].dtype)}
    from paper_2608_17402_gb300 import moevie
    case, out = s["case"], s["out"]
    if op == "join":
        moevie.moevie_residual_norm(s["norms"], s["r"], s["f"], s["ws"], out=out)
        got = {"r": out.r, "u": out.u, "stats_pre": out.stats_pre, "stats_post": out.stats_post}
        if case["save"]:
            got["kept_r"] = moevie.moevie_checkpoint_load(out.save_r, out=s["kept_r"])
            got["kept_f"] = moevie.moevie_checkpoint_load(out.save_f, out=s["kept_f"])
        return got
    if op == "join-bwd":
        moevie.moevie_residual_norm_backward(s["norms"], s["dr"], s["du"], s["r"], s["f"], s["stats_pre"],
                                             s["stats_post"], s["ws"], out=out)
        return {n: getattr(out, n) for n in ("dr", "df", "dw_pre", "db_pre", "dw_post", "db_post", "dgate")}
    if op == "balance":
        moevie.moevie_balance_loss(s["s"], s["idx"], s["ws"], coef=s["coef"], score=case["score"], seg=s["seg"], out=out)
        return {"loss": out.loss, "counts": out.counts, "ds": out.ds}
    moevie.moevie_checkpoint_store(s["x"], out=s["ck"])
    return {"x": moevie.moevie_checkpoint_load(s["ck"], out=out)}


# ------------------------------------------------------------ work, 64 bits

def work(case):
    op, T = case["op"], case["T"]
    if op == "balance":
        E = case["E"]
        return {"bytes": 8 * T * E + 4 * T * case["k"] + 4 * case["G"] * E, "flops": 12 * T * E}
    n = T * case["d"]
    kept, res = 1 + 4 / BLOCK, 2 if case["res"] == "bf16" else 4
    if op == "keep":
        return {"bytes": n * (2 * res + 2 * kept), "flops": 6 * n}
    gates = case["d"] * case["G"] if case["gate"] else 0
    norms = (1 + (case["post"] != "none")) * case["d"] * (2 if case["bias"] else 1)
    if op == "join":   # with save: codes written, and read back in the rows' own types
        saved = 2 * 2 * kept + res + 2 if case["save"] else 0
        return {"bytes": n * (2 * res + 4 + saved) + 16 * T + 4 * (norms + gates), "flops": 16 * n}
    rows = 2 * kept if case["saved"] == "q8" else res + 2
    return {"bytes": n * (2 * res + 2 + (4 if case["du"] == "f32" else 2) + rows) + 16 * T + 8 * (norms + gates),
            "flops": 30 * n}


def _keep64(x):
    """The values that blocks of a row are kept as."""
    parts = []
    for b in x.to(torch.float64).split(BLOCK, dim=1):
        top = b.abs().max(dim=1, keepdim=True)[0]
        parts.append(torch.where(top >= 2.0 ** -110, torch.round(b * 127 / top) * top / 127, 0.0))
    return torch.cat(parts, dim=1)


def _rows_of_gate64(s):
    T, f64 = s["case"]["T"], torch.float64
    if s["gate"] is None:
        return torch.ones(1, 1, dtype=f64, device="cuda")
    if s["seg"] is None:
        return s["gate"].to(f64)
    where = torch.bucketize(torch.arange(T, device="cuda"), s["seg"][1:].long(), right=True)
    return s["gate"].to(f64)[where]


def _join64(s):
    case, f64 = s["case"], torch.float64
    d = case["d"]

    def norm(x, kind, w, b):
        mean = x.sum(1, keepdim=True) / d if kind == "layer" else torch.zeros_like(x[:, :1])
        z = x - mean
        rstd = torch.rsqrt(torch.einsum("td,td->t", z, z) / d + EPS).unsqueeze(1)
        y = torch.einsum("td,t,d->td", z, rstd[:, 0], w.to(f64))
        return y if b is None else y + b.to(f64), torch.cat([mean, rstd], 1)

    n, stats_post = s["f"].to(f64), None
    if case["post"] != "none":
        n, stats_post = norm(n, case["post"], s["w_post"], s["b_post"])
    r1 = torch.addcmul(case["alpha"] * s["r"].to(f64), _rows_of_gate64(s), n)
    u, stats_pre = norm(r1, case["pre"], s["w_pre"], s["b_pre"])
    out = {"r": r1, "u": u, "stats_pre": stats_pre, "stats_post": stats_post}
    if case["save"]:
        out["kept_r"], out["kept_f"] = _keep64(s["r"]), _keep64(s["f"])
    return out


def _join_back64(s):
    case, f64 = s["case"], torch.float64
    G, T, d = case["G"], case["T"], case["d"]

    def rows(x):
        if case["saved"] != "q8":
            return x.to(f64)
        return torch.cat([c.to(f64) * x[1][:, i:i + 1].to(f64) for i, c in enumerate(x[0].split(BLOCK, dim=1))], dim=1)

    def unit(x, stats):
        return (x - stats[:, :1].to(f64)) * stats[:, 1:].to(f64)

    def through(g, z, stats, kind):   # d(norm's output / weight) -> d(its input)
        along = torch.einsum("td,td->t", g, z)[:, None] / d
        level = g.sum(1, keepdim=True) / d if kind == "layer" else 0.0
        return stats[:, 1:].to(f64) * (g - along * z - level)

    du, gate = s["du"].to(f64), _rows_of_gate64(s)
    z1, f = unit(rows(s["r"]), s["stats_pre"]), rows(s["f"])
    total = s["dr"].to(f64) + through(du * s["w_pre"].to(f64), z1, s["stats_pre"], case["pre"])
    gated = total * gate
    out = {"dr": total * case["alpha"], "dw_pre": torch.einsum("td,td->d", du, z1), "df": gated,
           "db_pre": du.sum(0) if s["b_pre"] is not None else None, "dw_post": None, "db_post": None, "dgate": None}
    n = f
    if case["post"] != "none":
        z2 = unit(f, s["stats_post"])
        w, b = s["w_post"].to(f64), s["b_post"]
        out["df"] = through(gated * w, z2, s["stats_post"], case["post"])
        out["dw_post"] = torch.einsum("td,td->d", gated, z2)
        out["db_post"] = gated.sum(0) if b is not None else None
        n = z2 * w if b is None else z2 * w + b.to(f64)
    if s["gate"] is not None:
        ends = [0, T] if s["seg"] is None else s["seg"].tolist()
        out["dgate"] = torch.stack([torch.einsum("td,td->d", total[a:b], n[a:b]) for a, b in zip(ends, ends[1:])])
    return out


def _balance64(s):
    case, f64 = s["case"], torch.float64
    T, E, k = case["T"], case["E"], case["k"]
    ends = [0, T] if s["seg"] is None else s["seg"].tolist()
    loss, counts, ds = torch.zeros(1, dtype=f64, device="cuda"), [], []
    for a, b in zip(ends, ends[1:]):
        n = torch.bincount(s["idx"][a:b].reshape(-1).long(), minlength=E)
        counts.append(n)
        z = s["s"][a:b].to(f64)
        c = n.to(f64) * (s["coef"] * E / (k * T * max(1, b - a)))
        score = torch.softmax(z, 1) if case["score"] == "softmax" else torch.special.expit(z)
        total = score.sum(1, keepdim=True)
        p = score / total
        mean = p @ c
        loss += mean.sum()
        rate = (c - mean[:, None]) / total   # dL/dscore
        ds.append(score * rate * (1.0 if case["score"] == "softmax" else 1 - score))
    return {"loss": loss, "counts": torch.stack(counts).to(torch.int32), "ds": torch.cat(ds)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "join":
        return _join64(s)
    if case["op"] == "join-bwd":
        return _join_back64(s)
    if case["op"] == "balance":
        return _balance64(s)
    return {"x": _keep64(s["x"])}
