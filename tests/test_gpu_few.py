"""moevie_moe_few (the whole layer for 1 to 64 tokens) against the oracle: selection
bit-exact, gates to fp32, y element by element.

Tolerance of y: the products are those of bf16 operands accumulated in 32 bits, hidden
activations keep at least 16 significant bits, so all that is left is the rounding of y to
bf16: half an ulp, 2^-9 relative to each element, and fp32 accumulation errors that are
small against the RMS of y.  REL = 2.5e-3 (2-norm; bf16 rounding alone gives 1.7e-3) and
|err| <= 2^-8 |y| + 1e-3 RMS."""
import numpy as np
import pytest
import torch

import oracle
import workloads
from paper_2608_17402_gb300 import moevie
from tests._gpu import check_status, dev, dev_bf16, layer_to_device, to_np_f64

pytestmark = pytest.mark.gpu

REL = 2.5e-3


def _few(lay, W=None, x=None):
    c = lay.cfg
    if W is None:
        x, W = layer_to_device(lay)
    ws = moevie.FewWorkspace(c.T, c.d, c.E, c.k, c.h, c.h_s)
    y, idx, gate = moevie.moevie_moe_few(W, x, ws, routing=True)
    check_status(ws)
    return y, idx, gate


def _want(lay):
    c = lay.cfg
    return oracle.forward_tokens(lay.x, lay.Wr, lay.b, lay.W1, lay.W2, c.k, lay.Ws1, lay.Ws2, c.lam,
                                 W3=lay.W3, Ws3=lay.Ws3)


def _close(y, want):
    got = to_np_f64(y)
    assert np.all(np.isfinite(got))
    rms = np.sqrt(np.mean(want ** 2))
    err = np.abs(got - want)
    assert np.linalg.norm(err) <= REL * np.linalg.norm(want), np.linalg.norm(err) / np.linalg.norm(want)
    worst = (err - 2.0 ** -8 * np.abs(want)).max()
    assert worst <= 1e-3 * rms, (worst, rms)


def _check(lay):
    y, idx, gate = _few(lay)
    want, widx, wgate, _ = _want(lay)
    assert np.array_equal(idx.cpu().numpy(), widx)
    assert np.abs(gate.cpu().numpy() - wgate).max() <= 1e-5
    _close(y, want)


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("T,d,E,k,h,hs", [
    (1, 8, 1, 1, 1, 0), (1, 64, 4, 2, 13, 5), (2, 96, 3, 3, 40, 0), (3, 72, 33, 5, 200, 100),
    (1, 768, 16, 2, 768, 0), (5, 256, 64, 8, 129, 65), (17, 136, 12, 4, 64, 192), (33, 520, 40, 7, 136, 0),
    (64, 128, 8, 8, 96, 96), (64, 200, 200, 1, 72, 0), (16, 1664, 64, 8, 416, 0), (7, 1280, 31, 7, 854, 854),
    (48, 1024, 1024, 32, 24, 8), (64, 64, 2, 1, 300, 600)])
def test_few_matches_oracle(T, d, E, k, h, hs, act):
    cfg = workloads.small_config(T=T, d=d, E=E, k=k, h=h, h_s=hs, lam=0.75, seed=T * 31 + h, act=act)
    _check(workloads.make_layer(cfg))


def test_few_agrees_with_the_batch_forward():
    """The same selection and, to the batch path's bf16 hidden activations, the same y."""
    lay = workloads.make_layer(workloads.small_config(T=64, d=512, E=32, k=4, h=256, h_s=256, seed=4))
    x, W = layer_to_device(lay)
    y, idx, _ = _few(lay, W, x)
    c = lay.cfg
    ws = moevie.Workspace(c.T, c.d, c.E, c.k, c.h, c.h_s)
    y2, rt = moevie.moevie_moe_forward(W, x, ws, routing=True)
    assert torch.equal(idx, rt["idx"])
    d = (y.float() - y2.float()).norm() / y2.float().norm()
    assert float(d) <= 1e-2


def test_few_tokens_do_not_depend_on_their_company():
    """Selection and gates of a token are the same alone and among others, y too up to the
    order of its sums; a repeated call gives the same bits."""
    lay = workloads.make_layer(workloads.small_config(T=40, d=384, E=24, k=3, h=160, h_s=64, seed=9))
    x, W = layer_to_device(lay)
    y, idx, gate = _few(lay, W, x)
    ws = moevie.FewWorkspace(64, 384, 24, 3, 160, 64)   # sized for more tokens than are passed
    for T in (40, 1, 9, 40):
        for t0 in (0, 40 - T):
            y1, i1, g1 = moevie.moevie_moe_few(W, x[t0:t0 + T].contiguous(), ws, routing=True)
            assert torch.equal(i1, idx[t0:t0 + T])
            assert torch.allclose(g1, gate[t0:t0 + T], rtol=1e-5, atol=0)
            assert torch.allclose(y1.float(), y[t0:t0 + T].float(), rtol=2.0 ** -7, atol=1e-3)
            if T == 40:
                assert torch.equal(y1, y) and torch.equal(g1, gate)
    check_status(ws)


def test_few_exact_ties_and_near_ties():
    """Duplicate router columns tie exactly (the lowest id wins); columns one part in 2^23
    apart differ by less than 32-bit sums resolve, and the exact order decides."""
    lay = workloads.make_layer(workloads.small_config(T=32, d=1024, E=48, k=4, h=32, seed=13))
    lay.b[:] = 0.0
    rng = np.random.default_rng(3)
    for e in range(0, 48, 3):
        lay.Wr[:, e + 1] = lay.Wr[:, e]
        bump = rng.integers(0, 2, size=1024).astype(np.float32)
        lay.Wr[:, e + 2] = lay.Wr[:, e] * (1 + bump * np.float32(2.0 ** -23))
    _check(lay)
    lay.Wr[:] = 0.0   # every expert ties
    _, idx, gate = _few(lay)
    assert np.array_equal(idx.cpu().numpy(), np.tile(np.arange(4, dtype=np.int32), (32, 1)))
    assert np.allclose(gate.cpu().numpy(), 0.25)


def test_few_extreme_logits_and_bias():
    """Saturated sigmoids (keys equal to the last bit of 64) and biases that alone decide."""
    lay = workloads.make_layer(workloads.small_config(T=6, d=64, E=10, k=3, h=24, seed=2))
    lay.Wr[:] *= 1000.0
    _check(lay)
    lay.Wr[:] *= 1e-6
    lay.b[:] = np.linspace(-5, 5, 10, dtype=np.float32)
    _check(lay)


def test_few_nonfinite_tokens_stay_alone():
    """A token holding NaN or infinity gets valid ids and a NaN output; the others are as
    without it."""
    lay = workloads.make_layer(workloads.small_config(T=9, d=128, E=12, k=3, h=48, h_s=16, seed=6))
    x, W = layer_to_device(lay)
    y, idx, _ = _few(lay, W, x)
    x2 = x.clone()
    x2[2, 5] = float("nan")
    x2[7, 0] = float("inf")
    y2, i2, _ = _few(lay, W, x2)
    ok = [t for t in range(9) if t not in (2, 7)]
    assert torch.equal(y2[ok], y[ok]) and torch.equal(i2[ok], idx[ok])
    assert torch.isnan(y2[[2, 7]].float()).any(1).all()
    ids = i2.cpu().numpy()
    assert ids.min() >= 0 and ids.max() < 12 and np.all(np.diff(ids, axis=1) > 0)


def test_few_unselected_experts_are_not_touched():
    """Experts that no token selects may hold anything."""
    lay = workloads.make_layer(workloads.small_config(T=4, d=96, E=20, k=2, h=40, seed=8))
    lay.b[10:] = -10.0
    x, W = layer_to_device(lay)
    y, idx, _ = _few(lay, W, x)
    assert int(idx.max()) < 10
    W.W1[10:] = float("nan")
    W.W2[10:] = float("nan")
    y2, _, _ = _few(lay, W, x)
    assert torch.equal(y, y2)


def test_few_capture_streams_and_reuse():
    """One workspace for layers of other sizes in turn, another stream, and a CUDA graph whose
    replays follow the input buffer."""
    lay = workloads.make_layer(workloads.small_config(T=8, d=256, E=16, k=4, h=96, seed=21))
    x, W = layer_to_device(lay)
    want, _, _ = _few(lay, W, x)
    ws = moevie.FewWorkspace(64, 512, 64, 8, 256, 256)
    small = workloads.make_layer(workloads.small_config(T=3, d=64, E=5, k=2, h=24, h_s=8, seed=22))
    xs, Ws = layer_to_device(small)
    wants, _, _ = _few(small, Ws, xs)
    for _ in range(3):
        assert torch.equal(moevie.moevie_moe_few(W, x, ws), want)
        assert torch.equal(moevie.moevie_moe_few(Ws, xs, ws), wants)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = moevie.moevie_moe_few(W, x, ws)
    s.synchronize()
    assert torch.equal(y, want)
    buf, out = x.clone(), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moevie.moevie_moe_few(W, buf, ws, y=out)
    for shift in (0, 3):
        buf.copy_(x.roll(shift, 0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want.roll(shift, 0))
    check_status(ws)


def test_few_refusals():
    lay = workloads.make_layer(workloads.small_config(T=2, d=64, E=4, k=2, h=16, seed=1))
    x, W = layer_to_device(lay)
    ws = moevie.FewWorkspace(2, 64, 4, 2, 16)
    with pytest.raises(ValueError):
        moevie.moevie_moe_few(W, x.float(), ws)
    with pytest.raises(ValueError):
        moevie.moevie_moe_few(W, x[:, :56].contiguous(), ws)
    with pytest.raises(moevie.MoevieError) as e:
        moevie.moevie_moe_few(W, x.repeat(40, 1), ws)
    assert e.value.code == 2
    big = x.repeat(32, 1)
    with pytest.raises(moevie.MoevieError) as e:
        moevie.moevie_moe_few(W, big, ws)
    assert e.value.code == 3
    n0 = moevie.moevie_launch_count()
    assert moevie.moevie_moe_few(W, x[:0], ws).shape == (0, 64)
    assert moevie.moevie_launch_count() == n0


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("T,d,E,k,h,hs", [
    (16, 200, 6, 3, 72, 40), (17, 200, 6, 3, 72, 40), (1, 328, 9, 9, 328, 328), (64, 1000, 90, 6, 520, 264),
    (60, 72, 33, 32, 130, 0), (31, 1032, 5, 2, 65, 129), (2, 2048, 300, 1, 8, 8)])
def test_few_odd_blocks(T, d, E, k, h, hs, act):
    """Odd numbers of K blocks, token counts around the one-copy bound of 16, wide and narrow
    tiles of both activations, entries of more than 32 tokens."""
    cfg = workloads.small_config(T=T, d=d, E=E, k=k, h=h, h_s=hs, lam=1.5, seed=T * 17 + d, act=act)
    _check(workloads.make_layer(cfg))
