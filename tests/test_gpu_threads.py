"""Calls from host threads other than the first."""
import os
import subprocess
import sys
import threading

import pytest
import torch

import workloads
from paper_2608_17402_gb300 import moevie
from tests._gpu import check_status, layer_to_device

pytestmark = pytest.mark.gpu


def _in_a_thread(call):
    """What ``call`` returns in a new host thread, whose first CUDA work it is."""
    got = []

    def run():
        try:
            got.append((call(), None))
        except Exception as e:   # to the test's own thread
            got.append((None, e))
    t = threading.Thread(target=run)
    t.start()
    t.join()
    torch.cuda.synchronize()
    result, error = got[0]
    assert error is None, error
    return result


@pytest.mark.parametrize("T", [3, 40])
def test_a_new_thread_may_begin_with_the_layer(T):
    lay = workloads.make_layer(workloads.small_config(T=T, d=128, E=8, k=2, h=72, h_s=40, seed=3))
    x, W = layer_to_device(lay)
    c = lay.cfg
    few = moevie.FewWorkspace(c.T, c.d, c.E, c.k, c.h, c.h_s)
    fwd = moevie.Workspace(c.T, c.d, c.E, c.k, c.h, c.h_s)
    want, want_fwd = moevie.moevie_moe_few(W, x, few), moevie.moevie_moe_forward(W, x, fwd)
    y = torch.empty_like(x)   # (an allocation in the thread could be its first CUDA work)
    assert torch.equal(_in_a_thread(lambda: moevie.moevie_moe_few(W, x, few, y=y)), want)
    assert torch.equal(_in_a_thread(lambda: moevie.moevie_moe_forward(W, x, fwd, y=y)), want_fwd)
    check_status(few)
    check_status(fwd)


@pytest.mark.parametrize("N,r,c", [(3, 200, 264), (70, 40, 304), (2, 64, 512), (4, 16, 96)])
def test_a_new_thread_may_begin_with_an_update(N, r, c):
    """Tiles, tiles of two matrices, a cluster for each, thin matrices."""
    U = torch.randn(N, r, c, device="cuda")
    ws = moevie.OrthoWorkspace(N, r, c)
    want = moevie.moevie_orthogonalize(U, ws)
    O = torch.zeros_like(want)
    assert torch.equal(_in_a_thread(lambda: moevie.moevie_orthogonalize(U, ws, out=O)), want)
    W, M = torch.randn(N, r, c, device="cuda"), torch.zeros(N, r, c, device="cuda")
    W2, M2 = W.clone(), M.clone()
    moevie.moevie_muon_update(W, M, U, ws, lr=0.1)
    _in_a_thread(lambda: moevie.moevie_muon_update(W2, M2, U, ws, lr=0.1))
    assert torch.equal(W, W2) and torch.equal(M, M2)
    check_status(ws)


ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import threading
import torch
import workloads
from paper_2608_17402_gb300 import moevie
from tests._gpu import layer_to_device

lay = workloads.make_layer(workloads.small_config(T=12, d=128, E=8, k=2, h=72, h_s=40, seed=3))
x, W = layer_to_device(lay)
U = torch.randn(3, 200, 264, device="cuda")
V = torch.randn(2, 40, 300, device="cuda")
c = lay.cfg
n = 8
spaces = [(moevie.FewWorkspace(c.T, c.d, c.E, c.k, c.h, c.h_s), moevie.Workspace(c.T, c.d, c.E, c.k, c.h, c.h_s),
           moevie.OrthoWorkspace(3, 200, 264), moevie.OrthoWorkspace(2, 40, 300)) for _ in range(n)]
torch.cuda.synchronize()
start, got, failed = threading.Barrier(n), [None] * n, []

def work(i):
    try:
        few, fwd, a, b = spaces[i]
        start.wait()
        got[i] = (moevie.moevie_moe_few(W, x, few), moevie.moevie_moe_forward(W, x, fwd),
                  moevie.moevie_orthogonalize(U, a), moevie.moevie_orthogonalize(V, b))
    except Exception as e:
        failed.append(repr(e))

threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
for t in threads:
    t.start()
for t in threads:
    t.join()
torch.cuda.synchronize()
assert not failed, failed
for g in got[1:]:
    assert all(torch.equal(p, q) for p, q in zip(g, got[0]))
for s in spaces:
    assert all(moevie.moevie_get_device_status(w)[0] == 0 for w in s)
print("threads agree")
"""


def test_first_calls_of_several_host_threads():
    """Several host threads make their first calls at once, in a process of its own: per-device set-up
    (kernel attributes, the tensor-map encoder, cluster counts) is shared between them.  Work goes
    to one stream, so only the host side runs at the same time."""
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "threads agree" in r.stdout
