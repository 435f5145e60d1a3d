"""The block's steps where memory that nothing wrote would show: padding in buffers that the calls make themselves, calls
without rows, the columns between rows of logits.  Fresh memory is filled with NaN here (with the largest whole number
for integer types), as torch does on request."""
import contextlib

import pytest
import torch

import workloads
from paper_2608_17402_gb300 import moevie
from tests._gpu import check_status, layer_to_device

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@contextlib.contextmanager
def fresh_memory_is_nan():
    was = torch.are_deterministic_algorithms_enabled()
    torch.use_deterministic_algorithms(True)
    try:
        assert torch.utils.deterministic.fill_uninitialized_memory
        yield
    finally:
        torch.use_deterministic_algorithms(was)


def _layer(T, d, E, k, h, **kw):
    lay = workloads.make_layer(workloads.small_config(T, d, E, k, h, seed=T + d, **kw))
    return layer_to_device(lay)[1]


def _steps(W, seg, r, dr, du, n0, n1, k):
    """The first norm, the layer, its balance loss, the join behind it, and all of it back, on buffers that the calls
    make."""
    T, d = r.shape
    E, h = W.W_r.shape[1], W.W2.shape[1]
    G = seg.numel() - 1
    norms = [moevie.ResidualNorm(d, seg=seg, **p) for p in (n0, n1)]
    fwd, bwd = moevie.Workspace(T, d, E, k, h), moevie.BackwardWorkspace(T, d, E, k, h)
    nws, bws = moevie.ResidualNormWorkspace(T, d, G), moevie.BalanceWorkspace(T, E, k, G)
    with fresh_memory_is_nan():
        first = moevie.moevie_residual_norm(norms[0], r, None, nws, save=True)
        f, rt = moevie.moevie_moe_forward(W, first.u, fwd, routing=True)
        s = moevie.moevie_router_logits(first.u, W.W_r, fwd)
        bal = moevie.moevie_balance_loss(s, rt["idx"], bws, 5.0, seg=seg)
        second = moevie.moevie_residual_norm(norms[1], r, f, nws, save=True)
        g1 = moevie.moevie_residual_norm_backward(norms[1], dr, du, second.r, second.save_f, second.stats_pre,
                                                  second.stats_post, nws)
        gl = moevie.moevie_moe_backward(W, first.u, g1.df, rt["idx"], bwd, ds=bal.ds)
        g0 = moevie.moevie_residual_norm_backward(norms[0], g1.dr, gl["dx"], first.save_r, None, first.stats_pre, None, nws)
    for ws in (fwd, bwd, nws, bws):
        check_status(ws)
    rows = {"u0": first.u, "r1": second.r, "u1": second.u, "dr1": g1.dr, "df": g1.df, "ds": bal.ds, "dr0": g0.dr,
            "dx": gl["dx"]}
    for n, ck in (("r0", first.save_r), ("r", second.save_r), ("f", second.save_f)):
        rows["codes " + n], rows["scale " + n] = ck.codes, ck.scale
        rows["kept " + n] = moevie.moevie_checkpoint_load(ck, F32)
    for n, o in (("0", first), ("1", second)):
        rows |= {m + n: getattr(o, m) for m in ("stats_pre", "stats_post") if getattr(o, m) is not None}
    sums = {"loss": bal.loss, "counts": bal.counts, **{n: gl[n] for n in gl if n != "dx"},
            **{n + "0": getattr(g0, n) for n in ("dw_pre", "db_pre")},
            **{n + "1": getattr(g1, n) for n in ("dw_pre", "dw_post", "db_post", "dgate")}}
    return rows, sums


@pytest.mark.parametrize("res", [BF, F32])
@pytest.mark.parametrize("front,behind", [(0, 21), (5, 0), (7, 40), (300, 300)])
def test_padding_through_the_layer_on_the_calls_own_buffers(front, behind, res):
    """Rows of padding, which hold NaN in every input, do not change what the others give, and are zeros in everything
    that the calls make: the same steps without the padding give the same, up to the order of fp32 sums over 300 rows
    (each term's share of 300 * 2^-24 < 2e-5; the sums of their sizes are some 20 times the results in the norm)."""
    n, d, E, k, h, G = 300, 136, 8, 2, 64, 3
    T = front + n + behind
    W = _layer(n, d, E, k, h)
    g = torch.Generator(device="cuda")
    g.manual_seed(front + behind)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    n0 = dict(pre="layer", w_pre=1 + normal(d, std=0.2), b_pre=normal(d, std=0.1))
    n1 = dict(pre="rms", post="layer", w_pre=1 + normal(d, std=0.2), w_post=1 + normal(d, std=0.2),
              b_post=normal(d, std=0.1), gate=normal(G, d, std=0.5), residual_scale=0.75)
    ends = torch.tensor([0, 77, 77, n], dtype=torch.int32, device="cuda")
    inputs = [normal(n, d).to(res), normal(n, d, std=1e-2).to(res), normal(n, d, std=1e-2)]
    padded = [torch.full((T, d), float("nan"), dtype=t.dtype, device="cuda") for t in inputs]
    for t, p in zip(inputs, padded):
        p[front:front + n] = t
    want_rows, want = _steps(W, ends, *inputs, n0, n1, k)
    got_rows, got = _steps(W, ends + front, *padded, n0, n1, k)
    for name, t in got_rows.items():
        outside = torch.cat([t[:front], t[front + n:]]).float()
        assert not bool(outside.any()), f"{name}: padding holds something"
    for name in ("u0", "r1", "u1", "codes r0", "codes r", "scale r0", "scale r", "stats_pre0"):
        assert torch.equal(got_rows[name][front:front + n], want_rows[name]), name
    assert torch.equal(got["counts"], want["counts"])
    for name, t in want.items():
        err = float((got[name].double() - t.double()).norm())
        assert err <= 1e-3 * float(t.double().norm()), (name, err)


def test_without_rows_the_weights_gradients_are_zeros():
    d, G = 264, 3
    w = {n: torch.ones(d, device="cuda") for n in ("w_pre", "b_pre", "w_post", "b_post")}
    norms = moevie.ResidualNorm(d, "layer", "rms", gate=torch.ones(G, d, device="cuda"),
                                seg=torch.zeros(G + 1, dtype=torch.int32, device="cuda"), **w)
    ws = moevie.ResidualNormWorkspace(0, d, G)
    rows, stats = torch.empty(0, d, device="cuda"), torch.empty(0, 2, device="cuda")
    for stream in (None, torch.cuda.Stream()):
        with fresh_memory_is_nan():
            g = moevie.moevie_residual_norm_backward(norms, rows, rows, rows, rows.to(BF), stats, stats, ws, stream=stream)
        torch.cuda.synchronize()
        assert g.dr.shape == g.df.shape == (0, d)
        for name in ("dw_pre", "db_pre", "dw_post", "db_post", "dgate"):
            assert not bool(getattr(g, name).any()), name
        # and into buffers of the caller's
        for name in ("dw_pre", "db_pre", "dw_post", "db_post", "dgate"):
            getattr(g, name).fill_(3.0)
        torch.cuda.synchronize()
        moevie.moevie_residual_norm_backward(norms, rows, rows, rows, rows.to(BF), stats, stats, ws, out=g, stream=stream)
        torch.cuda.synchronize()
        for name in ("dw_pre", "db_pre", "dw_post", "db_post", "dgate"):
            assert not bool(getattr(g, name).any()), name
    check_status(ws)


@pytest.mark.parametrize("act,h_s", [("gelu", 0), ("swiglu", 64)])
def test_without_tokens_the_layers_gradients_are_zeros(act, h_s):
    d, E, k, h = 64, 8, 2, 40
    W = _layer(4, d, E, k, h, act=act, h_s=h_s)
    ws = moevie.BackwardWorkspace(4, d, E, k, h, h_s=h_s, swiglu=act == "swiglu")
    x = torch.empty(0, d, dtype=BF, device="cuda")
    idx = torch.empty(0, k, dtype=torch.int32, device="cuda")
    for ds in (None, torch.empty(0, E, device="cuda")):
        with fresh_memory_is_nan():
            g = moevie.moevie_moe_backward(W, x, x, idx, ws, ds=ds)
        for name, t in g.items():
            assert not bool(t.any()), name
    check_status(ws)


@pytest.mark.parametrize("T,d,E", [(1, 8, 1), (70, 64, 33), (300, 512, 100), (70, 64, 129), (300, 512, 129), (1000, 64, 200),
                                   (1000, 1024, 200), (33, 768, 510), (64, 64, 1000), (500, 1536, 1000), (3, 264, 1021)])
def test_columns_between_rows_of_logits_are_zeros(T, d, E):
    """Rows lie E rounded up to a multiple of 32 apart; K of the product is split (many small widths) or not."""
    W = _layer(T, d, E, 1, 16)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    x = torch.randn(T, d, generator=g, device="cuda").to(BF)
    E32 = -(-E // 32) * 32
    with fresh_memory_is_nan():
        ws = moevie.Workspace(T, d, E, 1, 16)
        s = moevie.moevie_router_logits(x, W.W_r, ws)
    check_status(ws)
    whole = s.as_strided((T, E32), (E32, 1))
    assert not bool(whole[:, E:].any())
    assert bool(torch.isfinite(s).all())
    mine = torch.full((T, E32), float("nan"), device="cuda")
    moevie.moevie_router_logits(x, W.W_r, ws, s=mine)
    assert torch.equal(mine, whole)


@pytest.mark.parametrize("T", [1, 2, 7, 300, 5000])
def test_clear_padding(T):
    """Rows of 4 to 6656 bytes at every address of 4 bytes; ends of runs outside the rows, or that do not ascend, stay
    within the buffers."""
    gen = torch.Generator()
    gen.manual_seed(T)
    for ends in ((0, T), (0, 0), (T, T), (T // 2, T), (0, T // 2), (T // 3, 2 * T // 3), (-5, T + 5), (T // 2, -1), (T + 3, T + 9)):
        lo = min(max(ends[0], 0), T)
        hi = min(max(ends[1], lo), T)
        seg = torch.tensor([ends[0], (lo + hi) // 2, ends[1]], dtype=torch.int32, device="cuda")
        whole, want, rows = [], [], []
        for i, words in enumerate((1, 2, 3, 5, 8, 31, 33, 1664)):
            off = i % 4
            t = torch.randint(1, 1 << 30, (off + T * words + 9,), generator=gen, dtype=torch.int32).cuda()
            w = t.clone()
            part = w[off:off + T * words].view(T, words)
            part[:lo] = 0
            part[hi:] = 0
            whole.append(t)
            want.append(w)
            rows.append(t[off:off + T * words].view(T, words))
        moevie.moevie_clear_padding(seg, *rows)
        for t, w in zip(whole, want):
            assert torch.equal(t, w), ends


def test_clear_padding_on_a_stream_and_in_a_graph():
    seg = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    x, y = torch.ones(50, 33, device="cuda"), torch.ones(50, 8, dtype=torch.int8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            moevie.moevie_clear_padding(seg, x, None, y)
    torch.cuda.synchronize()
    seg.copy_(torch.tensor([5, 50], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert not bool(x[:5].any()) and not bool(y[:5].any()) and bool((x[5:] == 1).all()) and bool((y[5:] == 1).all())
    seg.copy_(torch.tensor([5, 48], dtype=torch.int32))
    torch.cuda.synchronize()
    moevie.moevie_clear_padding(seg, x, y, stream=s)
    torch.cuda.synchronize()
    assert not bool(x[48:].any()) and not bool(y[48:].any()) and bool((x[5:48] == 1).all()) and bool((y[5:48] == 1).all())


def test_clear_padding_of_large_buffers():
    """More than 2^31 bytes in front of the runs."""
    T, words = (1 << 31) // 1664 + 2000, 1664
    x = torch.ones(T, words, dtype=torch.int8, device="cuda")
    seg = torch.tensor([T - 7, T - 3], dtype=torch.int32, device="cuda")
    moevie.moevie_clear_padding(seg, x)
    assert not bool(x[:T - 7].any()) and bool((x[T - 7:T - 3] == 1).all()) and not bool(x[T - 3:].any())
