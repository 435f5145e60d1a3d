"""moevie_residual_norm and its backward against their formulas in 64 bits (the backward's by automatic
differentiation of the forward's formula), at the widths, runs and types where they can go wrong."""
import threading

import pytest
import torch

from paper_2608_17402_gb300 import moevie
from tests._block import EPS, group_of_rows, join64, near, q8_64, runs, stats64
from tests._gpu import check_status

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
SENTINEL = 777.0


class Case:
    """Inputs of one block; `pad` rows in front of and behind the runs."""

    def __init__(self, T, d, res=BF, pre="layer", post="layer", bias=True, gate=True, G=1, pad=(0, 0), alpha=0.75,
                 join=True, seed=0):
        gen = torch.Generator()
        gen.manual_seed(seed + 1000 * d + T)
        self.T, self.d, self.res, self.join = T, d, res, join

        def normal(*shape, std=1.0):
            return (torch.randn(*shape, generator=gen) * std).cuda()

        self.seg = runs(T, G, gen, pad) if G > 1 or pad != (0, 0) else None
        self.rows = group_of_rows(T, self.seg) if self.seg is not None else torch.zeros(T, dtype=torch.int64, device="cuda")
        self.p = {"pre": pre, "post": post, "alpha": alpha, "w_pre": 1 + normal(d, std=0.3) if pre else None,
                  "b_pre": normal(d, std=0.2) if pre and bias else None,
                  "w_post": 1 + normal(d, std=0.3) if post else None,
                  "b_post": normal(d, std=0.2) if post and bias else None,
                  "gate": normal(G, d, std=0.5) if gate else None}
        self.r = (normal(T, d) * torch.exp(normal(d, std=0.7)) + 0.2).to(res)
        self.f = (normal(T, d) * torch.exp(normal(T, 1, std=0.5))).to(BF) if join else None
        self.dr, self.du = normal(T, d, std=1e-2).to(res), normal(T, d, std=1e-2)
        self.norms = moevie.ResidualNorm(d, seg=self.seg, residual_scale=alpha, eps=EPS,
                                         **{k: v for k, v in self.p.items() if k != "alpha"})
        self.ws = moevie.ResidualNormWorkspace(T, d, G)
        self.live = self.rows >= 0

    def p64(self, grad=False):
        return {k: v.double().requires_grad_(grad) if isinstance(v, torch.Tensor) else v for k, v in self.p.items()}

    def out(self, save=False):
        """Buffers full of a value that rows of padding must keep."""
        o = moevie.ResidualNormOut.empty(self.norms, self.T, self.res, save, self.join)
        for t in (o.r, o.u, o.stats_pre, o.stats_post):
            if t is not None:
                t.fill_(SENTINEL)
        return o


def check_forward(c, o):
    live = c.live
    f64 = c.f.double()[live] if c.join else None
    r64 = c.r.double()[live]
    p = c.p64()
    r1, u = join64(p, r64, f64, c.rows[live])
    if c.join:
        n, _ = join64({**p, "alpha": 0.0}, r64, f64, c.rows[live])
        near(o.r[live], r1, r64.abs() + n.abs().amax(1, keepdim=True), "r")
        if c.p["post"]:
            near(o.stats_post[live], stats64(f64, c.p["post"]),
                 torch.cat([f64.abs().mean(1, keepdim=True), stats64(f64, c.p["post"])[:, 1:]], 1), "stats_post")
    if c.p["pre"]:
        s = stats64(r1, c.p["pre"])
        # the mean's error is that of a sum of |r1|; the norm's that of r1 itself times 1 / deviation
        near(o.stats_pre[live], s, torch.cat([r1.abs().mean(1, keepdim=True), s[:, 1:]], 1), "stats_pre")
        z = (r1.abs().amax(1, keepdim=True) * s[:, 1:]) * p["w_pre"].abs()
        near(o.u[live], u, z + (p["b_pre"].abs() if p["b_pre"] is not None else 0), "u")
    for t in (o.r, o.u, o.stats_pre, o.stats_post):
        if t is not None:
            assert bool((t[~live] == SENTINEL).all()), "padding was written"
    check_status(c.ws)


WIDTHS = [(1, 8), (1, 768), (1, 8192), (2, 256), (3, 264), (5, 248), (17, 1000), (64, 512), (33, 1024), (257, 768),
          (40, 1664), (9, 2048), (7, 4096), (6, 4104), (5, 8192), (1300, 136), (700, 1280)]


@pytest.mark.parametrize("res", [BF, F32])
@pytest.mark.parametrize("T,d", WIDTHS)
def test_forward_widths(T, d, res):
    c = Case(T, d, res)
    check_forward(c, moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, out=c.out()))


KINDS = [("rms", "rms", True, True), ("rms", None, False, True), ("layer", "rms", False, False), (None, "layer", True, True),
         ("layer", None, True, False), (None, None, False, True), ("rms", "layer", False, True)]


@pytest.mark.parametrize("pre,post,bias,gate", KINDS)
@pytest.mark.parametrize("res", [BF, F32])
def test_forward_kinds(pre, post, bias, gate, res):
    c = Case(37, 520, res, pre, post, bias, gate)
    check_forward(c, moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, out=c.out()))


RUNS = [(50, 264, 4, (0, 0)), (50, 264, 4, (3, 5)), (1000, 72, 90, (0, 17)), (300, 768, 1, (10, 20)), (41, 4104, 5, (1, 2)),
        (2000, 1664, 63, (0, 0)), (5, 8, 9, (0, 0)), (30, 512, 3, (15, 15))]


@pytest.mark.parametrize("T,d,G,pad", RUNS)
def test_forward_runs_and_padding(T, d, G, pad):
    c = Case(T, d, F32, "layer", "layer", G=G, pad=pad)
    c.r[~c.live] = float("nan")   # padding is not read
    c.f[~c.live] = float("inf")
    check_forward(c, moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, out=c.out()))


@pytest.mark.parametrize("T,d", [(1, 768), (300, 1288), (20, 8192), (77, 8), (9, 4104)])
@pytest.mark.parametrize("res", [BF, F32])
def test_saved_checkpoints_are_those_of_store(T, d, res):
    c = Case(T, d, res)
    o = moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, out=c.out(save=True))
    check_forward(c, o)
    for got, x in ((o.save_r, c.r), (o.save_f, c.f)):
        want = moevie.moevie_checkpoint_store(x)
        assert torch.equal(got.codes, want.codes) and torch.equal(got.scale, want.scale)


@pytest.mark.parametrize("res", [BF, F32])
@pytest.mark.parametrize("T,d", [(20, 1288), (3, 8192), (1, 8)])
def test_first_norm_of_rows_and_of_their_checkpoint(T, d, res):
    """f = None: u = N_pre(r), r whole or in 8 bits."""
    c = Case(T, d, res, join=False)
    check_forward(c, moevie.moevie_residual_norm(c.norms, c.r, None, c.ws, out=c.out()))
    ck = moevie.moevie_checkpoint_store(c.r)
    c.r = moevie.moevie_checkpoint_load(ck, F32)
    check_forward(c, moevie.moevie_residual_norm(c.norms, ck, None, c.ws, out=c.out()))


def test_in_place_on_the_stream_itself():
    c = Case(300, 1032, F32)
    want = moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws)
    o = c.out()
    o.r = c.r
    moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, out=o)
    assert torch.equal(o.r, want.r) and torch.equal(o.u, want.u)


def test_rows_with_nan_or_infinity_stay_by_themselves():
    c = Case(12, 520, F32)
    want = moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws)
    c.r[3, 5] = float("nan")
    c.f[7, 100] = float("inf")
    got = moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws)
    keep = torch.tensor([i not in (3, 7) for i in range(12)])
    assert torch.equal(got.u[keep], want.u[keep]) and torch.equal(got.r[keep], want.r[keep])
    assert bool(torch.isnan(got.u[3]).all()) and bool(torch.isnan(got.u[7]).any())


def test_rows_of_zeros_and_of_one_value():
    """eps alone is under the root: a constant row's layer norm is its bias."""
    c = Case(4, 264, F32, post="layer", pre="rms", alpha=1.0, gate=False)
    c.r.zero_()
    c.f[0] = 0
    c.f[1] = 3.0
    o = moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, out=c.out())
    check_forward(c, o)
    assert torch.equal(o.r[0], c.p["b_post"]) and torch.equal(o.r[1], c.p["b_post"])


# ------------------------------------------------------------------ backward

def backward64(c, r, f, stats_pre, stats_post, du, dr1):
    """Gradients by automatic differentiation of the formula at rows r, f, and the sizes that their sums run over."""
    live, rows = c.live, c.rows[c.live]
    p = c.p64(grad=True)
    r1 = r.double()[live].requires_grad_()
    f64 = f.double()[live].requires_grad_() if f is not None else None
    total = dr1.double()[live] if dr1 is not None else torch.zeros_like(r1)
    scale = {"total": total.abs()}
    got = {}
    if p["pre"]:
        s = stats_pre.double()[live]
        # by the formula, with the given statistics
        w = p["w_pre"].detach()
        x1, a = (r1.detach() - s[:, :1]) * s[:, 1:], du.double()[live] * w
        back = a - x1 * (a * x1).mean(1, keepdim=True) - (a.mean(1, keepdim=True) if p["pre"] == "layer" else 0)
        total = total + s[:, 1:] * back
        scale["total"] = scale["total"] + s[:, 1:] * (a.abs() + (1 + x1.abs()) * (a * x1).abs().mean(1, keepdim=True)
                                                      + a.abs().mean(1, keepdim=True))
        got["dw_pre"], got["db_pre"] = (du.double()[live] * x1).sum(0), du.double()[live].sum(0)
        scale["dw_pre"] = (du.double()[live].abs() * (1 + x1.abs())).sum(0)
        scale["db_pre"] = du.double()[live].abs().sum(0)
    got["dr"] = c.p["alpha"] * total if f is not None else total
    if f is not None:
        s = stats_post.double()[live] if p["post"] else None
        x2 = (f64.detach() - s[:, :1]) * s[:, 1:] if p["post"] else f64.detach()
        gate = p["gate"].detach()[rows] if p["gate"] is not None else torch.ones_like(x2)
        h, hs = gate * total, gate.abs() * scale["total"]
        n = x2 if not p["post"] else x2 * p["w_post"].detach() + (p["b_post"].detach() if p["b_post"] is not None else 0)
        G = 1 if c.seg is None else c.seg.numel() - 1
        got["dgate"] = torch.zeros(G, c.d, dtype=torch.float64, device="cuda").index_add_(0, rows, total * n)
        scale["dgate"] = torch.zeros(G, c.d, dtype=torch.float64, device="cuda").index_add_(
            0, rows, scale["total"] * (1 + n.abs() + (p["b_post"].detach().abs() if p["b_post"] is not None else 0)))
        got["df"], scale["df"] = h, hs
        if p["post"]:
            w = p["w_post"].detach()
            cc = h * w
            got["df"] = s[:, 1:] * (cc - x2 * (cc * x2).mean(1, keepdim=True)
                                    - (cc.mean(1, keepdim=True) if p["post"] == "layer" else 0))
            ccs = hs * w.abs()
            scale["df"] = s[:, 1:] * (ccs + (1 + x2.abs()) * (ccs * x2.abs()).mean(1, keepdim=True)
                                      + ccs.mean(1, keepdim=True))
            got["dw_post"], got["db_post"] = (h * x2).sum(0), h.sum(0)
            scale["dw_post"], scale["db_post"] = (hs * (1 + x2.abs())).sum(0), hs.sum(0)
    scale["dr"] = scale["total"]
    return got, scale


def check_backward(c, du=None, q8=False, dr1=True):
    du = c.du if du is None else du
    join = c.join
    r1, f = c.r, c.f   # any rows will do for r1
    st_pre = stats64(r1.double(), c.p["pre"]).float() if c.p["pre"] else None
    st_post = stats64(f.double(), c.p["post"]).float() if join and c.p["post"] else None
    R, Fr = r1, f
    if q8:
        R = moevie.moevie_checkpoint_store(r1)
        r1 = moevie.moevie_checkpoint_load(R, F32)
        if join:
            Fr = moevie.moevie_checkpoint_store(f)
            f = moevie.moevie_checkpoint_load(Fr, F32)
    o = moevie.ResidualNormGrads.empty(c.norms, c.T, c.res, join)
    for t in (o.dr, o.df):
        if t is not None:
            t.fill_(SENTINEL)
    d1 = c.dr if dr1 else None
    moevie.moevie_residual_norm_backward(c.norms, d1, du if c.p["pre"] else None, R if c.p["pre"] else None, Fr, st_pre,
                                         st_post, c.ws, out=o)
    want, scale = backward64(c, r1, f, st_pre, st_post, du, d1)
    for name in ("dr", "df"):
        t = getattr(o, name)
        if t is not None:
            near(t[c.live], want[name], scale[name], name)
            assert bool((t[~c.live] == SENTINEL).all()), "padding was written"
    for name in ("dw_pre", "db_pre", "dw_post", "db_post", "dgate"):
        t = getattr(o, name)
        if t is not None:
            near(t, want[name], scale[name], name)
    check_status(c.ws)
    return o


@pytest.mark.parametrize("res", [BF, F32])
@pytest.mark.parametrize("T,d", WIDTHS)
def test_backward_widths(T, d, res):
    check_backward(Case(T, d, res))


@pytest.mark.parametrize("pre,post,bias,gate", KINDS)
@pytest.mark.parametrize("res", [BF, F32])
def test_backward_kinds(pre, post, bias, gate, res):
    check_backward(Case(37, 520, res, pre, post, bias, gate))


@pytest.mark.parametrize("T,d,G,pad", RUNS)
def test_backward_runs_and_padding(T, d, G, pad):
    c = Case(T, d, F32, "layer", "layer", G=G, pad=pad)
    c.r[~c.live] = c.du[~c.live] = c.dr[~c.live] = float("nan")
    c.f[~c.live] = float("inf")
    check_backward(c)


@pytest.mark.parametrize("res", [BF, F32])
@pytest.mark.parametrize("du", [BF, F32])
@pytest.mark.parametrize("T,d", [(1, 768), (130, 1288), (7, 8192), (500, 72)])
def test_backward_from_checkpoints(T, d, du, res):
    c = Case(T, d, res, G=3 if T > 3 else 1)
    check_backward(c, du=c.du.to(du), q8=True)


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("T,d,G,gate", [(130, 1288, 1, True), (40, 2304, 6, True), (9, 8192, 1, False), (500, 72, 40, True)])
def test_backward_without_a_norm_behind_the_layer(T, d, G, gate, bias, q8):
    check_backward(Case(T, d, BF, "layer", None, bias, gate, G), q8=q8)


@pytest.mark.parametrize("d", [1032, 2056])
@pytest.mark.parametrize("post", ["rms", None])
def test_backward_of_wanted_gradients_alone(post, d):
    """Each gradient wanted by itself has the bits of all wanted together, but for sums formed beside others."""
    c = Case(70, d, F32, "layer", post, G=3)
    want = check_backward(c)
    st = stats64(c.r.double(), "layer").float(), stats64(c.f.double(), post).float() if post else None
    for name in ("dw_pre", "db_pre", "dgate", *(("dw_post", "db_post") if post else ())):
        o = moevie.ResidualNormGrads(torch.empty_like(want.dr), torch.empty_like(want.df))
        setattr(o, name, torch.full_like(getattr(want, name), SENTINEL))
        moevie.moevie_residual_norm_backward(c.norms, c.dr, c.du, c.r, c.f, *st, c.ws, out=o)
        assert torch.equal(o.dr, want.dr) and torch.equal(o.df, want.df)
        assert torch.equal(getattr(o, name), getattr(want, name)), name
    check_status(c.ws)


@pytest.mark.parametrize("T,d", [(130, 1288), (300, 72), (40, 2056), (9, 8072)])
def test_backward_from_checkpoints_after_rows_of_nan(T, d):
    """Rows that end within a warp's first block of a checkpoint: what an earlier call left on chip does not enter."""
    bad = Case(4000, 2048, F32, "rms", "rms")
    for t in (bad.r, bad.f, bad.dr, bad.du):
        t.fill_(float("nan"))
    c = Case(T, d, BF)
    want = check_backward(c, q8=True)
    r, f = moevie.moevie_checkpoint_store(c.r), moevie.moevie_checkpoint_store(c.f)
    good = [stats64(t.double(), "layer").float() for t in (c.r, c.f)]
    st = torch.full((4000, 2), float("nan"), device="cuda")
    for call in (lambda: moevie.moevie_residual_norm(bad.norms, bad.r, bad.f, bad.ws),
                 lambda: moevie.moevie_residual_norm_backward(bad.norms, bad.dr, bad.du, bad.r, bad.f, st, st, bad.ws)):
        got = moevie.ResidualNormGrads.empty(c.norms, T, BF)
        call()
        moevie.moevie_residual_norm_backward(c.norms, c.dr, c.du, r, f, *good, c.ws, out=got)
        for name in ("dr", "df", "dw_pre", "db_pre", "dw_post", "db_post", "dgate"):
            assert torch.equal(getattr(got, name), getattr(want, name)), name


def test_backward_of_the_first_norm():
    for q8 in (False, True):
        for dr1 in (False, True):
            check_backward(Case(61, 1032, F32, join=False), q8=q8, dr1=dr1)


def test_backward_in_place_and_without_weights_gradients():
    c = Case(200, 1032, BF)
    want = check_backward(c)
    st = [stats64(t.double(), "layer").float() for t in (c.r, c.f)]
    o = moevie.ResidualNormGrads(c.dr, torch.empty_like(want.df))
    moevie.moevie_residual_norm_backward(c.norms, c.dr, c.du, c.r, c.f, *st, c.ws, out=o)
    assert torch.equal(o.dr, want.dr) and torch.equal(o.df, want.df)


def test_formula_against_autograd_and_differences():
    """The backward's formula (backward64) is the derivative of the forward's: against automatic differentiation, and
    against differences along a random direction."""
    for pre, post, bias, gate in KINDS:
        c = Case(6, 40, F32, pre, post, bias, gate, G=2, pad=(1, 0))
        live, rows = c.live, c.rows[c.live]
        leaves = {"r": c.r.double()[live], "f": c.f.double()[live], **{k: v for k, v in c.p64().items()
                                                                     if isinstance(v, torch.Tensor)}}

        def loss(v):
            r1, u = join64({**c.p64(), **v}, v["r"], v["f"], rows)
            out = (r1 * c.dr.double()[live]).sum()
            return out if u is None else out + (u * c.du.double()[live]).sum()

        v = {k: t.clone().requires_grad_() for k, t in leaves.items()}
        loss(v).backward()
        r1 = join64(c.p64(), leaves["r"], leaves["f"], rows)[0]
        full = torch.zeros(c.T, c.d, dtype=torch.float64, device="cuda")
        full[live] = r1
        st_pre = stats64(full, pre) if pre else None
        st_post = stats64(c.f.double(), post) if post else None
        got, _ = backward64(c, full, c.f, st_pre, st_post, c.du, c.dr)
        for name, t in v.items():
            have = got["d" + name]
            assert float((have - t.grad).norm()) <= 1e-9 * float(t.grad.norm() + 1), name
        torch.manual_seed(1)
        h = 1e-5
        step = {k: torch.randn_like(t) for k, t in leaves.items()}
        slope = (loss({k: t + h * step[k] for k, t in leaves.items()}) - loss({k: t - h * step[k] for k, t in leaves.items()})) / (2 * h)
        along = sum(float((got["d" + k] * step[k]).sum()) for k in leaves)
        assert abs(float(slope) - along) <= 1e-6 * (1 + abs(along))


def test_a_block_forward_and_backward_with_its_checkpoints():
    """Two joins as a training step uses them: the second one's call keeps what the backward of both reads."""
    T, d = 257, 776
    a, b = Case(T, d, F32, seed=1), Case(T, d, F32, "rms", "rms", seed=2)
    one = moevie.moevie_residual_norm(a.norms, a.r, a.f, a.ws, save=True)
    two = moevie.moevie_residual_norm(b.norms, one.r, b.f, b.ws, save=True)
    g2 = moevie.moevie_residual_norm_backward(b.norms, b.dr, b.du, two.r, two.save_f, two.stats_pre, two.stats_post, b.ws)
    g1 = moevie.moevie_residual_norm_backward(a.norms, g2.dr, a.du, two.save_r, one.save_f, one.stats_pre,
                                              one.stats_post, a.ws)
    # against the same rows kept whole: what differs is the checkpoints' rounding, at most amax / 254 of a value
    w1 = moevie.moevie_residual_norm_backward(a.norms, g2.dr, a.du, one.r, a.f, one.stats_pre, one.stats_post, a.ws)
    for name in ("dr", "df", "dw_pre", "dw_post", "dgate"):
        x, y = getattr(g1, name).double(), getattr(w1, name).double()
        assert float((x - y).norm()) <= 0.05 * float(y.norm()), name
    back = moevie.moevie_residual_norm(a.norms, two.save_r, None, a.ws)   # the layer's input formed again
    assert float((back.u.double() - one.u.double()).norm()) <= 0.02 * float(one.u.double().norm())
    for c in (a, b):
        check_status(c.ws)


def test_same_bits_again_on_a_stream_and_in_a_graph():
    c = Case(900, 1288, BF, G=7)
    st = [stats64(t.double(), "layer").float() for t in (c.r, c.f)]

    def once(o, g):
        moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, out=o)
        moevie.moevie_residual_norm_backward(c.norms, c.dr, c.du, c.r, c.f, *st, c.ws, out=g)

    def bits(o, g):
        return [t.clone() for t in (o.r, o.u, o.stats_pre, o.stats_post, g.dr, g.df, g.dw_pre, g.db_pre, g.dw_post,
                                    g.db_post, g.dgate)]

    o, g = c.out(), moevie.ResidualNormGrads.empty(c.norms, c.T, BF)
    once(o, g)
    want = bits(o, g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        once(o, g)
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(bits(o, g), want))
        with torch.cuda.graph(graph, stream=s):
            once(o, g)
    for _ in range(3):
        for t in (o.u, g.dw_pre, g.dgate):
            t.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(bits(o, g), want))
    check_status(c.ws)


def test_calls_of_two_threads_on_two_streams():
    """Two programs at once, each with its workspace and stream, whose outputs the calls make."""
    cases = [Case(3000, 1288, BF, G=5), Case(800, 2304, F32, "rms", "layer", seed=1)]
    stats = [[stats64(t.double(), c.p[n]).float() for t, n in ((c.r, "pre"), (c.f, "post"))] for c in cases]

    def go(i, stream, out):
        c = cases[i]
        for _ in range(20):
            out[i] = (moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws, save=True, stream=stream),
                      moevie.moevie_residual_norm_backward(c.norms, c.dr, c.du, c.r, c.f, *stats[i], c.ws, stream=stream))

    want, got = [None, None], [None, None]
    for i in range(2):
        go(i, None, want)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=go, args=(i, torch.cuda.Stream(), got)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for (o, g), (wo, wg) in zip(got, want):
        assert torch.equal(o.u, wo.u) and torch.equal(o.r, wo.r) and torch.equal(o.save_f.codes, wo.save_f.codes)
        for name in ("dr", "df", "dw_pre", "dw_post", "dgate"):
            assert torch.equal(getattr(g, name), getattr(wg, name)), name
    for c in cases:
        check_status(c.ws)


def test_runs_that_do_not_ascend_are_a_device_error():
    for bad in ([0, 30, 20, 50], [-3, 10, 20, 50], [0, 10, 20, 51]):
        c = Case(50, 264, F32, G=3)
        c.norms.seg = torch.tensor(bad, dtype=torch.int32, device="cuda")
        moevie.moevie_residual_norm(c.norms, c.r, c.f, c.ws)
        assert moevie.moevie_get_device_status(c.ws)[0] == 6
        moevie.moevie_workspace_init(c.ws)
        st = [stats64(t.double(), "layer").float() for t in (c.r, c.f)]
        moevie.moevie_residual_norm_backward(c.norms, c.dr, c.du, c.r, c.f, *st, c.ws)
        assert moevie.moevie_get_device_status(c.ws)[0] == 6


def test_large_offsets():
    """Row offsets beyond 32 bits: the last rows of a stream of more than 2^32 bytes and 2^31 elements."""
    T, d = 270000, 8192
    free = torch.cuda.mem_get_info()[0]
    if free < 40e9:
        pytest.skip("needs 40 GB")
    r = torch.zeros(T, d, dtype=BF, device="cuda")
    f = torch.zeros(T, d, dtype=BF, device="cuda")
    tail = Case(5, d, BF, "rms", "rms", gate=False, seed=3)
    r[-5:], f[-5:] = tail.r, tail.f
    ws = moevie.ResidualNormWorkspace(T, d)
    o = moevie.moevie_residual_norm(tail.norms, r, f, ws, save=True)
    want = moevie.moevie_residual_norm(tail.norms, tail.r, tail.f, tail.ws, save=True)
    assert torch.equal(o.u[-5:], want.u) and torch.equal(o.r[-5:], want.r)
    assert torch.equal(o.save_r.codes[-5:], want.save_r.codes) and torch.equal(o.save_f.scale[-5:], want.save_f.scale)
    back = moevie.moevie_checkpoint_load(o.save_f)
    assert torch.equal(back[-5:], moevie.moevie_checkpoint_load(want.save_f))
    g = moevie.moevie_residual_norm_backward(tail.norms, r, f, o.r, f, o.stats_pre, o.stats_post, ws)
    g5 = moevie.moevie_residual_norm_backward(tail.norms, tail.r, tail.f, want.r, tail.f, want.stats_pre, want.stats_post,
                                              tail.ws)
    assert torch.equal(g.dr[-5:], g5.dr) and torch.equal(g.df[-5:], g5.df)


def test_what_is_refused():
    c = Case(4, 64, F32)
    run = moevie.moevie_residual_norm
    for bad in (dict(r=c.r.half()), dict(r=c.r[:, :56]), dict(f=c.f.float()), dict(f=c.f[:3]), dict(r=c.r.t()),
                dict(r=c.r.cpu())):
        with pytest.raises(ValueError):
            run(c.norms, bad.get("r", c.r), bad.get("f", c.f), c.ws)
    with pytest.raises(ValueError):
        run(moevie.ResidualNorm(64, w_pre=torch.ones(64, dtype=BF, device="cuda")), c.r, c.f, c.ws)
    with pytest.raises(ValueError):
        run(moevie.ResidualNorm(64, gate=torch.ones(2, 64, device="cuda")), c.r, c.f, c.ws)
    for norms, code in ((moevie.ResidualNorm(64, eps=0.0), 1), (moevie.ResidualNorm(64, residual_scale=float("nan")), 1),
                        (moevie.ResidualNorm(64, pre=None), 1)):
        with pytest.raises(moevie.MoevieError) as e:
            run(norms, c.r, None, c.ws)
        assert e.value.code == code
    with pytest.raises(moevie.MoevieError) as e:   # a checkpoint is no residual stream to add to
        run(c.norms, moevie.moevie_checkpoint_store(c.r), c.f, c.ws)
    assert e.value.code == 1
    small = moevie.ResidualNormWorkspace(1, 64)
    big = Case(1000, 64, F32)
    with pytest.raises(moevie.MoevieError) as e:
        run(big.norms, big.r, big.f, small)
    assert e.value.code == 3
