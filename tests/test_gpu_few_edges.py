"""moevie_moe_few where its CTAs wait on one another: a grid barrier that has timed out, parts that
are summed as they arrive.  Nothing here faults, traps or
hangs the GPU: the first test sets the mark that a timed-out barrier leaves."""
import pytest
import torch

import workloads
from paper_2608_17402_gb300 import moevie
from tests._gpu import check_status, layer_to_device

pytestmark = pytest.mark.gpu

ARRIVALS = 32   # byte of the status block at which the barriers' 64-bit count lies


@pytest.mark.parametrize("T", [4, 40])
def test_few_does_not_run_after_a_barrier_timed_out(T):
    """A timed-out barrier marks its count (the top bit), as that need not be a multiple of the
    grid any more: later calls leave their outputs as they were until the workspace is set up
    again.  T = 40 has two barriers a call."""
    lay = workloads.make_layer(workloads.small_config(T=T, d=256, E=16, k=4, h=96, h_s=32, seed=T))
    x, W = layer_to_device(lay)
    c = lay.cfg
    ws = moevie.FewWorkspace(c.T, c.d, c.E, c.k, c.h, c.h_s)
    want = moevie.moevie_moe_few(W, x, ws)
    check_status(ws)
    count = ws.buf[ARRIVALS:ARRIVALS + 8].view(torch.int64)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert count.item() == sms * (1 if T == 4 else 2)
    count += 5               # some CTAs of a broken-off launch,
    count |= -(1 << 63)      # and the mark
    y = torch.full_like(x, 7.0)
    for _ in range(3):
        moevie.moevie_moe_few(W, x, ws, y=y)
    assert torch.all(y == 7.0)
    assert count.item() < 0
    moevie.moevie_workspace_init(ws)
    for _ in range(2):
        assert torch.equal(moevie.moevie_moe_few(W, x, ws, y=y), want)
    check_status(ws)


@pytest.mark.parametrize("T", [2, 16, 64])
def test_few_gives_the_same_bits_every_time(T):
    """The sum over a token's parts starts as soon as the last of them is counted: a part read too
    early would be that of the call before, which here ran on other tokens."""
    lay = workloads.make_layer(workloads.small_config(T=T, d=520, E=24, k=6, h=200, h_s=136, seed=T + 1))
    x, W = layer_to_device(lay)
    c = lay.cfg
    ws = moevie.FewWorkspace(c.T, c.d, c.E, c.k, c.h, c.h_s)
    other = x.flip(0).neg().contiguous()
    want, want_other = moevie.moevie_moe_few(W, x, ws), moevie.moevie_moe_few(W, other, ws)
    got = []
    for _ in range(40):
        got.append((moevie.moevie_moe_few(W, x, ws), moevie.moevie_moe_few(W, other, ws)))
    assert all(torch.equal(a, want) and torch.equal(b, want_other) for a, b in got)
    check_status(ws)
