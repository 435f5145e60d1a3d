"""Plain 64-bit forms of the residual norms, the balance loss and the 8-bit checkpoints."""
import torch

EPS = 1e-6


def runs(T, G, gen, pad=(0, 0), empty=True):
    """Ends of G ragged runs within [pad[0], T - pad[1]], some of them empty."""
    lo, hi = pad[0], T - pad[1]
    cuts = torch.randint(lo, hi + 1, (G - 1,), generator=gen)
    if empty and G > 2:
        cuts[1] = cuts[0]
    return torch.cat([torch.tensor([lo]), torch.sort(cuts)[0], torch.tensor([hi])]).to(torch.int32).cuda()


def group_of_rows(T, seg):
    """The run of every row, -1 for padding."""
    out = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    ends = seg.tolist()
    for g, (a, b) in enumerate(zip(ends, ends[1:])):
        out[a:b] = g
    return out


def stats64(x, kind):
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    return torch.cat([mean, 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)], 1)


def norm64(x, kind, w, b):
    if kind is None:
        return x
    s = stats64(x, kind)
    y = (x - s[:, :1]) * s[:, 1:]
    y = y if w is None else y * w
    return y if b is None else y + b


def join64(p, r, f, rows):
    """(r1, u) of the parameters p (pre, post, weights, gate, alpha), all in 64 bits; rows: the run of every row."""
    r1 = r
    if f is not None:
        n = norm64(f, p["post"], p["w_post"], p["b_post"])
        r1 = p["alpha"] * r + (n if p["gate"] is None else p["gate"][rows] * n)
    return r1, None if p["pre"] is None else norm64(r1, p["pre"], p["w_pre"], p["b_pre"])


def q8_64(x):
    """Codes (as int8) and scales of the checkpoint of x [T, d], from its definition."""
    codes, scales = [], []
    for b in x.double().split(128, 1):
        top = b.abs().amax(1, keepdim=True)
        some = top >= 2.0 ** -110
        codes.append(torch.where(some, torch.round(127 * b / torch.where(some, top, 1.0)), 0.0).to(torch.int8))
        scales.append(torch.where(some, top.float() / torch.full_like(top, 127.0).float(), 0.0).float())
    return torch.cat(codes, 1), torch.cat(scales, 1)


def near(got, want, scale, what=""):
    """got against want (64 bits): half a step of got's type, and 2^-17 of `scale`, which is what 128 roundings of
    fp32 sums whose terms add up to `scale` in size can make."""
    eps = torch.finfo(got.dtype).eps / 2
    err = (got.double() - want).abs()
    most = eps * want.abs() + 2.0 ** -17 * scale + torch.finfo(got.dtype).smallest_normal
    bad = ~(err <= most)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {err.numel()} off, the worst {float((err / most).max()):.2f} times"
