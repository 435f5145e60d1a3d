"""moevie_moe_few on a workspace whose grid barrier has timed out.  Nothing here faults, traps or
hangs the GPU: the test sets the mark that a timed-out barrier leaves."""
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
