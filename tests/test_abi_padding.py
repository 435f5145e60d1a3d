"""C ABI of moevie_clear_padding, host side: what is refused, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2608_17402_gb300 import moevie

FAKE = 0x1000   # never read: every call ends before a launch
INVALID, UNSUPPORTED = 1, 2


class Buffer(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_void_p), ("row_bytes", ctypes.c_int64)]


@pytest.mark.parametrize("change,code", [
    (dict(T=0), 0), (dict(T=0, buffers=None, seg=None), 0), (dict(T=-1), INVALID), (dict(T=1 << 31), UNSUPPORTED),
    (dict(G=0), INVALID), (dict(G=(1 << 20) + 1), UNSUPPORTED), (dict(n=0), INVALID), (dict(n=17), UNSUPPORTED),
    (dict(buffers=None), INVALID), (dict(seg=None), INVALID), (dict(seg=FAKE + 2), INVALID),
    (dict(buffers=[(FAKE, 8), (None, 8)]), INVALID), (dict(buffers=[(FAKE, 8), (FAKE + 2, 8)]), INVALID),
    (dict(buffers=[(FAKE, 8), (FAKE, 0)]), INVALID), (dict(buffers=[(FAKE, 8), (FAKE, -4)]), INVALID),
    (dict(buffers=[(FAKE, 8), (FAKE, 6)]), INVALID), (dict(buffers=[(FAKE, 8), (FAKE, 1 << 31)]), INVALID)])
def test_arguments(change, code):
    v = dict(buffers=[(FAKE, 8), (FAKE, 12)], n=2, T=4, seg=FAKE, G=1)
    v.update(change)
    lib, n = moevie.load(), moevie.moevie_launch_count()
    b = None if v["buffers"] is None else (Buffer * 17)(*[Buffer(*x) for x in v["buffers"]])
    assert lib.moevie_clear_padding(b, v["n"], v["T"], v["seg"], v["G"], None) == code
    assert moevie.moevie_launch_count() == n


def test_refusals_of_the_binding(monkeypatch):
    calls = []
    monkeypatch.setattr(moevie, "_call", lambda name, *args: calls.append(args))
    monkeypatch.setattr(moevie, "_device", lambda: -1)
    monkeypatch.setattr(moevie, "_on", lambda stream, dev: None)
    seg = torch.tensor([1, 3], dtype=torch.int32)
    a, b = torch.zeros(4, 6), torch.zeros(4, 2, 3, dtype=torch.bfloat16)
    moevie.moevie_clear_padding(seg, a, None, b)
    assert len(calls) == 1 and calls[0][1:5] == (2, 4, seg.data_ptr(), 1)
    assert (Buffer * 2).from_buffer_copy(calls[0][0])[1].row_bytes == 12
    for bad in ((seg, a, torch.zeros(5, 6)), (seg, a.t()), (seg, torch.tensor(1.0)), (seg.long(), a), (seg, a[:, :2])):
        with pytest.raises(ValueError):
            moevie.moevie_clear_padding(*bad)
    moevie.moevie_clear_padding(seg)               # nothing to clear
    moevie.moevie_clear_padding(seg, None, a[:0])
    assert len(calls) == 1
