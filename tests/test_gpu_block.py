"""The block's steps together: the balance loss's gradient through the layer's backward, the router's logits, a
whole block against automatic differentiation in 64 bits, and the example."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import workloads
from paper_2608_17402_gb300 import moevie
from tests._block import EPS, join64, stats64
from tests._gpu import check_status, dev, dev_bf16, layer_to_device

pytestmark = pytest.mark.gpu


def _layer(T, d, E, k, h, **kw):
    lay = workloads.make_layer(workloads.small_config(T, d, E, k, h, seed=T + d, **kw))
    x, W = layer_to_device(lay)
    return lay, x, W


@pytest.mark.parametrize("T,d,E,k", [(1, 8, 1, 1), (130, 256, 16, 4), (77, 136, 33, 2), (300, 512, 129, 8), (64, 64, 1000, 3)])
def test_router_logits(T, d, E, k):
    """Against 64 bits: two bf16 pieces hold 2^-16 of a weight (each rounds by half a step), and the sum of d products
    is rounded to fp32 as often."""
    _, x, W = _layer(T, d, E, k, 16)
    ws = moevie.Workspace(T, d, E, k, 16)
    s = moevie.moevie_router_logits(x, W.W_r, ws)
    check_status(ws)
    assert s.shape == (T, E) and s.stride(0) % 32 == 0
    want = x.double() @ W.W_r.double()
    size = x.double().abs() @ W.W_r.double().abs()
    assert bool(((s.double() - want).abs() <= (2.0 ** -16 + d * 2.0 ** -24) * size + 1e-37).all())
    # the loss takes them as they lie
    idx = torch.sort(torch.topk(s, k, 1)[1], 1)[0].to(torch.int32)
    bws = moevie.BalanceWorkspace(T, E, k)
    got = moevie.moevie_balance_loss(s, idx, bws)
    want = moevie.moevie_balance_loss(s.contiguous(), idx, bws)
    assert torch.equal(got.counts, want.counts)
    assert abs(float(got.loss) - float(want.loss)) <= 1e-6 * abs(float(want.loss))


@pytest.mark.parametrize("T,d,E,k,h,h_s,act", [(300, 256, 16, 4, 128, 0, "gelu"), (130, 192, 31, 3, 64, 64, "swiglu"),
                                               (1, 64, 4, 2, 64, 0, "gelu"), (200, 96, 129, 3, 40, 0, "gelu")])
def test_gradient_of_all_logits(T, d, E, k, h, h_s, act):
    """With dy = 0 the layer's own gradient is nothing: what dx and dW_r get is ds W_r^T and x^T ds, the operands
    rounded to bf16 (2^-8 each at most)."""
    lay, x, W = _layer(T, d, E, k, h, h_s=h_s, act=act)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ds = torch.randn(T, E, generator=g, device="cuda")
    idx = torch.sort(torch.topk(ds, k, 1)[1], 1)[0].to(torch.int32)
    ws = moevie.BackwardWorkspace(T, d, E, k, h, h_s=h_s, swiglu=act == "swiglu")
    zero = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    out = moevie.moevie_moe_backward(W, x, zero, idx, ws, ds=ds)
    check_status(ws)
    ds64, wr, x64 = ds.double(), W.W_r.double(), x.double()
    for name, want, size in (("dx", ds64 @ wr.T, ds64.abs() @ wr.abs().T), ("dW_r", x64.T @ ds64, x64.abs().T @ ds64.abs())):
        err = (out[name].double() - want).abs()
        assert bool((err <= (2.0 ** -7 + 2.0 ** -16 + (T + E) * 2.0 ** -24) * size + 1e-30).all()), name
    for name in out:
        if name not in ("dx", "dW_r"):
            assert not bool(out[name].any()), name


def test_gradient_of_all_logits_beside_the_gates():
    """dy and ds together give what each gives alone, up to the rounding of their sum to bf16; rows of ds further
    apart are read as such, and without ds nothing changes."""
    T, d, E, k, h = 300, 256, 16, 4, 128
    lay, x, W = _layer(T, d, E, k, h)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    dy = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    wide = torch.randn(T, 40, generator=g, device="cuda") * 0.3
    ds = wide[:, :E]
    idx = torch.sort(torch.topk(torch.randn(T, E, generator=g, device="cuda"), k, 1)[1], 1)[0].to(torch.int32)
    ws = moevie.BackwardWorkspace(T, d, E, k, h)
    alone = moevie.moevie_moe_backward(W, x, dy, idx, ws)
    logits = moevie.moevie_moe_backward(W, x, torch.zeros_like(dy), idx, ws, ds=ds)
    both = moevie.moevie_moe_backward(W, x, dy, idx, ws, ds=ds)
    check_status(ws)
    for name in alone:
        a, b, c = (v[name].double() for v in (alone, logits, both))
        # three roundings of ds to bf16 where one was: 2^-8 of each part's size, which their norms bound
        assert float((c - a - b).norm()) <= 2.0 ** -8 * 2 * float(a.norm() + b.norm()) + 1e-30, name
    for name in ("dW1", "dW2"):
        assert float((both[name] - alone[name]).abs().max()) <= 1e-5 * float(alone[name].abs().max()), name


def test_a_block_against_automatic_differentiation():
    """r -> join -> layer -> join with the balance loss, every gradient against that of the formulas in 64 bits.  The
    library rounds u, f, df and the layer's GEMM operands to bf16: relative errors of 2^-8 at each of the four or
    five steps that a gradient passes, in the norm over many of them below 1e-2 (the layer's own tolerance)."""
    T, d, E, k, h = 256, 128, 8, 2, 64
    lay, _, W = _layer(T, d, E, k, h)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    r = normal(T, d)
    p0 = {"pre": "layer", "post": None, "alpha": 1.0, "w_pre": 1 + normal(d, std=0.2), "b_pre": normal(d, std=0.1),
          "w_post": None, "b_post": None, "gate": None}
    p1 = {"pre": "rms", "post": "layer", "alpha": 0.75, "w_pre": 1 + normal(d, std=0.2), "b_pre": None,
          "w_post": 1 + normal(d, std=0.2), "b_post": normal(d, std=0.1), "gate": normal(2, d, std=0.5)}
    seg = torch.tensor([0, 100, T], dtype=torch.int32, device="cuda")
    rows = (torch.arange(T, device="cuda") >= 100).long()
    dr2, du2, coef = normal(T, d), normal(T, d), 20.0
    n0, n1 = (moevie.ResidualNorm(d, seg=s, residual_scale=p["alpha"], eps=EPS,
                                  **{a: b for a, b in p.items() if a != "alpha"}) for p, s in ((p0, None), (p1, seg)))
    nws = moevie.ResidualNormWorkspace(T, d, 2)
    fwd, bwd, bal = moevie.Workspace(T, d, E, k, h), moevie.BackwardWorkspace(T, d, E, k, h), moevie.BalanceWorkspace(T, E, k, 2)

    first = moevie.moevie_residual_norm(n0, r, None, nws)
    f, rt = moevie.moevie_moe_forward(W, first.u, fwd, routing=True)
    s = moevie.moevie_router_logits(first.u, W.W_r, fwd)
    loss = moevie.moevie_balance_loss(s, rt["idx"], bal, coef, seg=seg)
    second = moevie.moevie_residual_norm(n1, r, f, nws)
    g1 = moevie.moevie_residual_norm_backward(n1, dr2, du2, second.r, f, second.stats_pre, second.stats_post, nws)
    gl = moevie.moevie_moe_backward(W, first.u, g1.df, rt["idx"], bwd, ds=loss.ds)
    g0 = moevie.moevie_residual_norm_backward(n0, g1.dr, gl["dx"], r, None, first.stats_pre, None, nws)
    for ws in (nws, fwd, bwd, bal):
        check_status(ws)

    leaves = {"r": r, "W_r": W.W_r, "W1": W.W1, "W2": W.W2, **{"0" + a: b for a, b in p0.items() if isinstance(b, torch.Tensor)},
              **{"1" + a: b for a, b in p1.items() if isinstance(b, torch.Tensor)}}
    leaves = {a: b.double().clone().requires_grad_() for a, b in leaves.items()}
    q0, q1 = ({**p, **{a[1:]: b for a, b in leaves.items() if a[0] == n}} for p, n in ((p0, "0"), (p1, "1")))
    _, u = join64(q0, leaves["r"], None, rows)
    idx = rt["idx"].long()
    logits = u @ leaves["W_r"]
    sig = torch.sigmoid(logits)
    gate = torch.gather(sig, 1, idx)
    gate = gate / gate.sum(1, keepdim=True)
    y = torch.zeros_like(u)
    for e in range(E):
        t, j = (idx == e).nonzero(as_tuple=True)
        a = torch.nn.functional.gelu(u[t] @ leaves["W1"][e])
        y = y.index_add(0, t, gate[t, j, None] * (a @ leaves["W2"][e]))
    r2, u2 = join64(q1, leaves["r"], y, rows)
    p = sig / sig.sum(1, keepdim=True)
    balance = 0.0
    for b in range(2):
        n = torch.bincount(idx[rows == b].reshape(-1), minlength=E).double()
        T_b = int((rows == b).sum())
        balance = balance + coef * T_b / T * (E * n / (k * T_b) * p[rows == b].mean(0)).sum()
    assert abs(float(loss.loss) - float(balance.detach())) <= 1e-3 * float(balance.detach())   # u in bf16
    ((r2 * dr2.double()).sum() + (u2 * du2.double()).sum() + balance).backward()
    got = {"r": g0.dr, "W_r": gl["dW_r"], "W1": gl["dW1"], "W2": gl["dW2"], "0w_pre": g0.dw_pre, "0b_pre": g0.db_pre,
           "1w_pre": g1.dw_pre, "1w_post": g1.dw_post, "1b_post": g1.db_post, "1gate": g1.dgate}
    assert sorted(got) == sorted(leaves)
    for name, t in leaves.items():
        rel = float((got[name].double() - t.grad).norm() / t.grad.norm())
        assert rel <= 1e-2, (name, rel)


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_block.py")
    spec = importlib.util.spec_from_file_location("train_block", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_example_runs():
    losses = _example().main(3)
    assert len(losses) == 3 and all(np.isfinite(losses))


def test_example_gradients():
    """Along the gradient of each of its tensors the example's loss moves as the gradient says: the difference
    quotient over a step that moves the loss by about a thousandth, where the stream is fp32 and what is rounded to
    bf16 (u, the layer's values: 2^-8 each, of 300,000 values) averages out: within 5 %.  The selection is held by
    the loss's own: tensors that move it (the routers, the first norm) are left to the test above."""
    example = _example()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    blocks = example.Blocks(gen)
    r, target = example.inputs(gen)
    _, dr, kept = blocks.loss(r, target)
    grads, layers = blocks.backward(dr, kept)
    last = blocks.norms[-1], grads[-1]
    for norms, g, names in ((*last, ("w_post", "gate")),):
        for name in names:
            w, dw = getattr(norms, name), getattr(g, "d" + name)
            step = 2e-3 / float((dw.double() ** 2).sum())
            keep = w.clone()
            ends = []
            for h in (step, -step):
                w.copy_(keep + h * dw)
                ends.append(float(blocks.loss(r, target)[0].double()))
            w.copy_(keep)
            slope = (ends[0] - ends[1]) / (2 * step)
            want = float((dw.double() ** 2).sum())
            assert abs(slope - want) <= 0.05 * want, (name, slope, want)
