"""What the binding of the block's steps checks of tensors that a program keeps from call to call, on the CPU: the
library's entry is replaced by one that does nothing, the device by the CPU's -1."""
import types

import pytest
import torch

from paper_2608_17402_gb300 import moevie

T, D, E, K, G = 4, 256, 8, 2, 3
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    calls = []
    monkeypatch.setattr(moevie, "_call", lambda name, *args: calls.append(name))
    monkeypatch.setattr(moevie, "_device", lambda: -1)
    monkeypatch.setattr(moevie, "_on", lambda stream, dev: None)
    return calls


WS = types.SimpleNamespace(buf=torch.zeros(16, dtype=torch.uint8), nbytes=16)


def norms():
    seg = torch.tensor([0, 1, 2, 4], dtype=torch.int32)
    w = {n: torch.ones(D) for n in ("w_pre", "b_pre", "w_post", "b_post")}
    return moevie.ResidualNorm(D, "layer", "rms", gate=torch.ones(G, D), seg=seg, **w)


def join():
    n = norms()
    out = moevie.ResidualNormOut.empty(n, T, F32, save=True, device="cpu")
    r, f = torch.zeros(T, D), torch.zeros(T, D, dtype=BF)
    held = {"norms." + a: (n, a) for a in ("w_pre", "b_pre", "w_post", "b_post", "gate", "seg")}
    held |= {"out." + a: (out, a) for a in ("r", "u", "stats_pre", "stats_post")}
    held |= {c + "." + a: (getattr(out, c), a) for c in ("save_r", "save_f") for a in ("codes", "scale")}
    return held, lambda: moevie.moevie_residual_norm(n, r, f, WS, out=out)


def join_back():
    n = norms()
    out = moevie.ResidualNormGrads.empty(n, T, F32, device="cpu")
    r, f = moevie.Checkpoint.empty(T, D, "cpu"), moevie.Checkpoint.empty(T, D, "cpu")
    s = torch.zeros(T, 2)
    dr, du = torch.zeros(T, D), torch.zeros(T, D)
    held = {"norms." + a: (n, a) for a in ("w_pre", "w_post", "gate", "seg")}
    held |= {"out." + a: (out, a) for a in ("dr", "df", "dw_pre", "db_pre", "dw_post", "db_post", "dgate")}
    held |= {c + "." + a: (ck, a) for c, ck in (("r", r), ("f", f)) for a in ("codes", "scale")}
    return held, lambda: moevie.moevie_residual_norm_backward(n, dr, du, r, f, s, s, WS, out=out)


def balance():
    out = moevie.BalanceOut.empty(T, E, device="cpu")
    s, idx = torch.zeros(T, E), torch.zeros(T, K, dtype=torch.int32)
    held = {"out." + a: (out, a) for a in ("loss", "counts", "ds")}
    return held, lambda: moevie.moevie_balance_loss(s, idx, WS, out=out)


def store():
    ck, x = moevie.Checkpoint.empty(T, D, "cpu"), torch.zeros(T, D)
    return {a: (ck, a) for a in ("codes", "scale")}, lambda: moevie.moevie_checkpoint_store(x, out=ck)


def load():
    ck, x = moevie.Checkpoint.empty(T, D, "cpu"), torch.zeros(T, D)
    return {a: (ck, a) for a in ("codes", "scale")}, lambda: moevie.moevie_checkpoint_load(ck, out=x)


def shorter(t):
    return t.flatten()[:-1].clone()


def other_type(t):
    return t.to(BF if t.dtype is F32 else torch.int16 if t.dtype is torch.int32 else torch.float16)


def apart(t):
    return torch.zeros(*t.shape, 2, dtype=t.dtype)[..., 0]


@pytest.mark.parametrize("change", [shorter, other_type, apart])
@pytest.mark.parametrize("make", [join, join_back, balance, store, load])
def test_a_kept_tensor_given_other_memory_is_refused(make, change, no_library):
    """`.data = ...`, which is also what a module's .to(), .half() and .bfloat16() do to its parameters."""
    held, call = make()
    call()
    assert no_library
    for name, (owner, field) in held.items():
        if change is apart and getattr(owner, field).numel() == 1:
            continue   # a single value has no strides
        t = getattr(owner, field)
        keep = t.data
        if change is other_type:
            # (.data takes tensors of the parameter's own type alone where autograd knows it; a module swaps it so)
            t.data = change(t)
        else:
            t.data = change(t)
        n = len(no_library)
        with pytest.raises(ValueError):
            call()
        assert len(no_library) == n, name
        t.data = keep
        call()


def test_parameters_of_a_module_that_changes_its_type(no_library):
    module = torch.nn.LayerNorm(D)
    n = moevie.ResidualNorm(D, "layer", w_pre=module.weight, b_pre=module.bias)
    r = torch.zeros(T, D)
    out = moevie.ResidualNormOut.empty(n, T, F32, join=False, device="cpu")
    moevie.moevie_residual_norm(n, r, None, WS, out=out)
    module.bfloat16()
    with pytest.raises(ValueError):
        moevie.moevie_residual_norm(n, r, None, WS, out=out)
    module.float()
    moevie.moevie_residual_norm(n, r, None, WS, out=out)
    assert len(no_library) == 2


def test_a_gate_of_other_runs_is_refused(no_library):
    held, call = join()
    call()
    n = held["norms.seg"][0]
    n.seg.data = torch.tensor([0, 4], dtype=torch.int32)   # one run, the gate still has three
    with pytest.raises(ValueError):
        call()
    n.gate.data = torch.ones(1, D)
    call()


@pytest.mark.parametrize("make", [join, join_back, balance, store, load])
def test_a_kept_tensor_without_memory_is_refused(make, no_library):
    """Storages that a program empties for a while; an address of none would be read as `not given`."""
    held, call = make()
    call()
    for name, (owner, field) in held.items():
        storage = getattr(owner, field).untyped_storage()
        size = storage.nbytes()
        storage.resize_(0)
        n = len(no_library)
        with pytest.raises(ValueError):
            call()
        assert len(no_library) == n, name
        storage.resize_(size)
        getattr(owner, field).zero_()
        call()


def test_the_type_of_a_stream_without_a_gradient(no_library):
    """dr = None: the stream's type is that of out.dr, else of r, and bf16 where neither says it."""
    n, s = moevie.ResidualNorm(D, "layer"), torch.zeros(T, 2)
    du, ck = torch.zeros(T, D), moevie.Checkpoint.empty(T, D, "cpu")
    out = moevie.ResidualNormGrads.empty(n, T, F32, join=False, device="cpu")

    def back(r, **kw):
        return moevie.moevie_residual_norm_backward(n, None, du, r, None, s, None, WS, **kw).dr.dtype
    assert back(ck, out=out) is F32 and back(torch.zeros(T, D)) is F32 and back(ck) is BF
    with pytest.raises(ValueError):
        moevie.moevie_residual_norm_backward(n, None, None, ck, None, s, None, WS)
