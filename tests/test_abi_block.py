"""C ABI of the residual norms, the checkpoints and the balance loss, host side: what is refused, before anything is
launched, and the workspaces' sizes.  No call here launches anything."""
import ctypes
import types

import pytest

from paper_2608_17402_gb300 import moevie
from paper_2608_17402_gb300.moevie import _Norms, _Rows

P = ctypes.c_void_p
FAKE = 0x1000   # never read: every call ends before a launch


@pytest.fixture(scope="module")
def lib():
    return moevie.load()


@pytest.fixture(autouse=True)
def nothing_is_launched(lib):
    n = moevie.moevie_launch_count()
    yield
    assert moevie.moevie_launch_count() == n


def norms(**kw):
    v = dict(d=64, pre=2, post=1, w_pre=FAKE, b_pre=0, w_post=FAKE, b_post=0, gate=FAKE, seg=0, G=1, residual_scale=1.0,
             eps=1e-6)
    v.update(kw)
    return _Norms(*v.values())


def forward(lib, n=None, r=(FAKE, None, 1), f=FAKE, T=4, r_out=FAKE, u=FAKE, stats=(FAKE, FAKE), save=(None,) * 4,
            ws=FAKE, ws_bytes=0):
    n = n or norms()
    return lib.moevie_residual_norm(ctypes.byref(n), ctypes.byref(_Rows(*r)), f, T, r_out, u, *stats, *save, ws, ws_bytes,
                                    None)


def backward(lib, n=None, dr1=FAKE, res=1, du=FAKE, du_f32=1, r1=(FAKE, None, 1), f=(FAKE, None, 0), stats=(FAKE, FAKE), T=4,
             dr=FAKE, df=FAKE, grads=(FAKE, None, FAKE, None, FAKE), ws=FAKE, ws_bytes=0):
    n = n or norms()
    return lib.moevie_residual_norm_backward(
        ctypes.byref(n), dr1, res, du, du_f32, ctypes.byref(_Rows(*r1)) if r1 else None,
        ctypes.byref(_Rows(*f)) if f else None, *stats, T, dr, df, *grads, ws, ws_bytes, None)


WORKSPACE, INVALID, UNSUPPORTED = 3, 1, 2


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("change,code", [
    (dict(), WORKSPACE), (dict(d=60), UNSUPPORTED), (dict(d=8200), UNSUPPORTED), (dict(d=8192), WORKSPACE), (dict(d=0), INVALID),
    (dict(d=-8), INVALID), (dict(pre=3), INVALID), (dict(post=-1), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(residual_scale=float("inf")), INVALID), (dict(residual_scale=float("nan")), INVALID),
    (dict(residual_scale=0.0), WORKSPACE), (dict(G=0), INVALID), (dict(G=2), INVALID), (dict(G=2, seg=FAKE), WORKSPACE),
    (dict(G=1 + (1 << 20), seg=FAKE), UNSUPPORTED), (dict(G=1 << 20, seg=FAKE), WORKSPACE), (dict(seg=FAKE + 2), INVALID), (dict(w_pre=FAKE + 8), INVALID),
    (dict(gate=FAKE + 4), INVALID), (dict(b_post=FAKE + 8), INVALID), (dict(post=0, w_post=0), None)])
def test_descriptions(lib, call, change, code):
    n = norms(**change)
    if code is None:   # no post norm: nothing of its weights' gradients
        assert forward(lib, n) == WORKSPACE
        assert backward(lib, n) == INVALID
        assert backward(lib, n, grads=(FAKE, None, None, None, FAKE)) == WORKSPACE
        return
    assert call(lib, n) == code


@pytest.mark.parametrize("args,code", [
    (dict(T=-1), INVALID), (dict(T=1 << 31), UNSUPPORTED), (dict(T=0, r=(None, None, 1), ws=None), 0),
    (dict(r=(None, None, 1)), INVALID), (dict(r=(FAKE + 8, None, 1)), INVALID), (dict(r=(FAKE, None, 3)), INVALID),
    (dict(r=(FAKE, FAKE, 2)), INVALID), (dict(r=(FAKE, None, 0)), WORKSPACE),
    (dict(r=(FAKE, FAKE, 2), f=None, r_out=None), WORKSPACE), (dict(r=(FAKE, None, 2), f=None, r_out=None), INVALID),
    (dict(r=(FAKE, FAKE, 2), f=None, r_out=None, save=(FAKE, FAKE, None, None)), INVALID),
    (dict(f=FAKE + 2), INVALID), (dict(r_out=None), INVALID), (dict(u=None), INVALID), (dict(u=FAKE + 8), INVALID),
    (dict(stats=(FAKE + 4, None)), INVALID), (dict(stats=(None, None)), WORKSPACE),
    (dict(save=(FAKE, None, None, None)), INVALID), (dict(save=(None, None, FAKE, FAKE + 2)), INVALID),
    (dict(save=(FAKE, FAKE, FAKE, FAKE)), WORKSPACE), (dict(f=None, save=(None, None, FAKE, FAKE)), INVALID),
    (dict(ws=None), INVALID), (dict(ws=FAKE + 8), INVALID)])
def test_forward_arguments(lib, args, code):
    assert forward(lib, **args) == code


def test_forward_without_a_norm_or_a_join(lib):
    none = norms(pre=0)
    assert forward(lib, none, u=None) == WORKSPACE      # the stream's last step
    assert forward(lib, none) == INVALID                # u without a norm
    assert forward(lib, none, f=None, u=None) == INVALID   # nothing to do


@pytest.mark.parametrize("args,code", [
    (dict(), WORKSPACE), (dict(T=0, dr=None), 0), (dict(res=2), INVALID), (dict(du_f32=-1), INVALID), (dict(dr=None), INVALID),
    (dict(dr1=None), WORKSPACE), (dict(du=None), INVALID), (dict(du=FAKE + 8), INVALID), (dict(r1=None), INVALID),
    (dict(r1=(FAKE, None, 0)), INVALID), (dict(r1=(FAKE, None, 0), res=0), WORKSPACE), (dict(r1=(FAKE, FAKE, 2)), WORKSPACE),
    (dict(f=(FAKE, None, 1)), INVALID), (dict(f=(FAKE, FAKE, 2)), WORKSPACE), (dict(f=None), INVALID),
    (dict(stats=(None, FAKE)), INVALID), (dict(stats=(FAKE, None)), INVALID), (dict(grads=(FAKE + 2,) + (None,) * 4), INVALID),
    (dict(grads=(None,) * 5), WORKSPACE), (dict(df=None), INVALID),
    (dict(df=None, f=None, stats=(FAKE, None), grads=(FAKE, FAKE, None, None, None)), WORKSPACE)])
def test_backward_arguments(lib, args, code):
    assert backward(lib, **args) == code


def test_backward_without_what_the_forward_left_out(lib):
    last = norms(pre=0)
    assert backward(lib, last, du=None, r1=None, stats=(None, FAKE), grads=(None, None, FAKE, FAKE, FAKE)) == WORKSPACE
    assert backward(lib, last, r1=None, stats=(None, FAKE), grads=(None,) * 5) == INVALID       # du without a norm
    assert backward(lib, last, dr1=None, du=None, r1=None, stats=(None, FAKE), grads=(None,) * 5) == INVALID
    assert backward(lib, norms(gate=0)) == INVALID                                               # dgate without a gate
    plain = norms(post=0, gate=0)
    assert backward(lib, plain, f=None, stats=(FAKE, None), grads=(FAKE,) + (None,) * 4) == WORKSPACE


@pytest.mark.parametrize("d", [8, 256, 264, 768, 1664, 4096, 8192])
def test_residual_workspace_serves_fewer_rows_and_runs(lib, d):
    out, prev = ctypes.c_size_t(0), 0
    for T in [0, 1, 2, 3, 7, 64, 151, 152, 153, 303, 608, 5000, 65536, 1 << 20]:
        before = 0
        for G in (1, 2, 63, 5000):
            assert lib.moevie_residual_norm_workspace_size(T, d, G, ctypes.byref(out)) == 0
            assert out.value >= before
            before = out.value
            if G == 1:
                assert out.value >= prev, T
                prev = out.value
    assert lib.moevie_residual_norm_workspace_size(1, d, 1, None) == INVALID
    assert lib.moevie_residual_norm_workspace_size(1, d + 4, 1, ctypes.byref(out)) == UNSUPPORTED
    assert lib.moevie_residual_norm_workspace_size(-1, d, 1, ctypes.byref(out)) == INVALID
    assert lib.moevie_residual_norm_workspace_size(1, d, 0, ctypes.byref(out)) == INVALID


@pytest.mark.parametrize("E,k", [(4, 2), (64, 8), (1024, 32)])
def test_balance_workspace_serves_fewer_tokens_and_runs(lib, E, k):
    out, prev = ctypes.c_size_t(0), 0
    for T in list(range(0, 70000, 997)) + [1 << 20]:
        before = 0
        for G in list(range(1, 40)) + [1000]:
            assert lib.moevie_balance_workspace_size(T, E, k, G, ctypes.byref(out)) == 0
            assert out.value >= before, (T, G)
            before = out.value
            if G == 1:
                assert out.value >= prev, T
                prev = out.value
    assert lib.moevie_balance_workspace_size(1, E, k, 0, ctypes.byref(out)) == INVALID
    assert lib.moevie_balance_workspace_size(1, E, E + 1, 1, ctypes.byref(out)) == UNSUPPORTED
    assert lib.moevie_balance_workspace_size(1, 2048, k, 1, ctypes.byref(out)) == UNSUPPORTED


@pytest.mark.parametrize("change,code", [
    (dict(), WORKSPACE), (dict(s=None), INVALID), (dict(s=FAKE + 2), INVALID), (dict(ld_s=15), INVALID), (dict(idx=None), INVALID),
    (dict(T=-1), INVALID), (dict(E=2000, ld_s=2000, ld_ds=2000), UNSUPPORTED), (dict(k=17), UNSUPPORTED), (dict(k=0), INVALID),
    (dict(T=1 << 30, k=4), UNSUPPORTED), (dict(G=2), INVALID), (dict(G=2, seg=FAKE), WORKSPACE), (dict(G=0), INVALID),
    (dict(G=1 << 20, seg=FAKE), WORKSPACE), (dict(G=(1 << 20) + 1, seg=FAKE), UNSUPPORTED), (dict(score=2), INVALID), (dict(coef=float("nan")), INVALID), (dict(loss=None), INVALID), (dict(counts=None), INVALID),
    (dict(ds=None), WORKSPACE), (dict(ds=None, ld_ds=0), WORKSPACE), (dict(ld_ds=8), INVALID), (dict(ds=FAKE, s=FAKE, ld_ds=20), INVALID),
    (dict(ws=None), INVALID)])
def test_balance_arguments(lib, change, code):
    v = dict(s=FAKE, ld_s=16, idx=FAKE, T=4, E=16, k=2, seg=None, G=1, score=1, coef=0.1, loss=FAKE, counts=FAKE,
             ds=2 * FAKE, ld_ds=16, ws=FAKE, ws_bytes=0)
    v.update(change)
    assert lib.moevie_balance_loss(*v.values(), None) == code


@pytest.mark.parametrize("call", ["store", "load"])
def test_checkpoint_arguments(lib, call):
    def run(a=FAKE, f32=1, T=4, d=64, b=FAKE, c=FAKE):
        if call == "store":
            return lib.moevie_checkpoint_store(a, f32, T, d, b, c, None)
        return lib.moevie_checkpoint_load(b, c, T, d, a, f32, None)
    assert run(T=0, a=None, b=None, c=None) == 0
    assert run(d=12) == UNSUPPORTED and run(T=1 << 31) == UNSUPPORTED
    for bad in (dict(a=None), dict(b=None), dict(c=None), dict(a=FAKE + 8), dict(b=FAKE + 8), dict(c=FAKE + 2), dict(f32=2),
                dict(T=-1), dict(d=0)):
        assert run(**bad) == INVALID, bad


def test_router_logits_and_balanced_backward(lib):
    from paper_2608_17402_gb300.moevie import _Layer
    assert lib.moevie_router_logits(FAKE, FAKE, 4, 16, 8, FAKE, FAKE, 0, None) == WORKSPACE
    assert lib.moevie_router_logits(None, FAKE, 4, 16, 8, FAKE, FAKE, 0, None) == INVALID
    assert lib.moevie_router_logits(FAKE, FAKE, 4, 16, 8, FAKE + 4, FAKE, 0, None) == INVALID
    assert lib.moevie_router_logits(FAKE, FAKE, 4, 12, 8, FAKE, FAKE, 0, None) == UNSUPPORTED
    assert lib.moevie_router_logits(None, None, 0, 16, 8, None, None, 0, None) == 0
    L = _Layer(16, 8, 2, 32, 0, FAKE, FAKE, FAKE, FAKE, 0, 0, 1.0)

    def back(ds=FAKE, ld=8, T=4):
        return lib.moevie_moe_backward_balanced(ctypes.byref(L), FAKE, FAKE, T, FAKE, ds, ld, *([FAKE] * 4), *([None] * 4),
                                                FAKE, 0, None)
    assert back() == WORKSPACE
    assert back(ds=None) == back(ds=FAKE + 2) == back(ld=7) == INVALID
    assert back(ds=None, T=0) == 0
    assert lib.moevie_moe_backward_balanced(None, FAKE, FAKE, 4, FAKE, FAKE, 8, *([FAKE] * 8), FAKE, 0, None) == INVALID


def test_refusals_of_the_binding():
    import torch
    n = moevie.ResidualNorm(64)
    with pytest.raises(ValueError):
        moevie._matrix(torch.zeros(4, 32), n.d, "r")
    with pytest.raises(ValueError):
        moevie._rows(torch.zeros(4, 64), (4, 64), torch.float32, 0, "r")   # not on the device
    with pytest.raises(ValueError):
        moevie._scratch(types.SimpleNamespace(buf=torch.zeros(4)), 0)      # nor its workspace
    with pytest.raises(KeyError):
        moevie._KINDS["batch"]
