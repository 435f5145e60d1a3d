"""8-bit checkpoints (moevie_checkpoint_store, moevie_checkpoint_load) against their definition in 64 bits: codes
bit for bit, scales and values by the rounding of one fp32 division and product."""
import pytest
import torch

from paper_2608_17402_gb300 import moevie
from tests._block import q8_64

pytestmark = pytest.mark.gpu


def _rows(T, d, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(T, d, generator=g, device="cuda") * torch.exp(2 * torch.randn(T, 1, generator=g, device="cuda"))
    return x.to(dtype)


def _check(x):
    ck = moevie.moevie_checkpoint_store(x)
    codes, scales = q8_64(x)
    assert torch.equal(ck.codes, codes)
    assert torch.equal(ck.scale, scales)   # one correctly rounded division
    want = codes.double() * scales.repeat_interleave(128, 1)[:, :x.shape[1]].double()
    got = moevie.moevie_checkpoint_load(ck, torch.float32)
    assert torch.equal(got, want.float())   # one rounding of the exact product
    half = moevie.moevie_checkpoint_load(ck, torch.bfloat16)
    assert torch.equal(half, want.float().to(torch.bfloat16))
    # at most half a code off, and the roundings of scale and value; in a block that is kept as zeros
    # (scale 0) the value itself, which by definition lies below 2^-110
    err = (got.double() - x.double()).abs()
    most = (0.5 + 127 * 2.0 ** -22) * scales.repeat_interleave(128, 1)[:, :x.shape[1]].double() + 2.0 ** -110
    assert bool((err <= most).all())
    return ck


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(1, 8), (1, 128), (3, 136), (7, 120), (197, 1288), (1000, 768), (33, 8192), (5, 16392),
                                 (2500, 264), (40000, 8), (1, 1664)])
def test_codes_scales_and_values(T, d, dtype):
    _check(_rows(T, d, dtype, T + d))


def test_borders_between_codes():
    """Values half-way between two codes go to the even one, whatever 127 / amax rounds to, and values a step to
    either side of half-way go where they belong."""
    rows = []
    for amax in (127.0, 254.0, 1.0, 3.0, 0.7, 1e-20, 1e20, 129.0, 1.0000001):
        a = torch.tensor(amax, dtype=torch.float32)
        half = (torch.arange(-126, 126, dtype=torch.float64) + 0.5) * a.double() / 127
        half = half.float()
        up, down = (torch.nextafter(half, torch.tensor(s)) for s in (float("inf"), float("-inf")))
        for v in (half, up, down):
            v = torch.cat([v, torch.zeros(2)])
            for part in v.split(127):
                rows.append(torch.cat([a.reshape(1), part]))
    x = torch.stack(rows).cuda()
    assert x.shape[1] == 128
    _check(x)
    _check(x.to(torch.bfloat16))


def test_blocks_of_zeros_and_of_tiny_values():
    x = torch.zeros(4, 256, device="cuda")
    x[1, 3] = 2.0 ** -110          # kept
    x[2, 7] = -(2.0 ** -111)       # below: kept as zeros
    x[3, 130] = 1e-40
    x[3, 0] = -1.5
    ck = _check(x)
    assert ck.codes[1, 3] == 127 and not ck.codes[2].any() and not ck.codes[3, 128:].any()
    assert not ck.scale[0].any() and ck.scale[1, 0] > 0 and ck.scale[2, 0] == 0 and ck.scale[3, 1] == 0


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_block_with_an_infinity_or_a_nan_comes_back_as_nan(bad, dtype):
    x = _rows(6, 392, dtype, 1)
    want = x.clone()
    x[2, 200] = bad
    got = moevie.moevie_checkpoint_load(moevie.moevie_checkpoint_store(x), dtype)
    clean = moevie.moevie_checkpoint_load(moevie.moevie_checkpoint_store(want), dtype)
    assert bool(torch.isnan(got[2, 128:256]).all())
    got[2, 128:256] = clean[2, 128:256] = 0
    assert torch.equal(got, clean)


def test_rows_behind_the_last_are_left_alone():
    x = _rows(10, 136, torch.bfloat16, 2)
    big = moevie.Checkpoint.empty(12, 136)
    big.codes.fill_(77)
    big.scale.fill_(5.0)
    out = moevie.Checkpoint(big.codes[:10], big.scale[:10])
    moevie.moevie_checkpoint_store(x, out=out)
    assert bool((big.codes[10:] == 77).all()) and bool((big.scale[10:] == 5.0).all())
    y = torch.full((12, 136), 3.0, device="cuda")
    moevie.moevie_checkpoint_load(out, out=y[:10])
    assert bool((y[10:] == 3.0).all())


def test_on_a_stream_and_in_a_graph():
    x = _rows(300, 1032, torch.bfloat16, 3)
    want = moevie.moevie_checkpoint_load(moevie.moevie_checkpoint_store(x))
    ck, y = moevie.Checkpoint.empty(300, 1032), torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        moevie.moevie_checkpoint_store(x, out=ck)
        moevie.moevie_checkpoint_load(ck, out=y)
        s.synchronize()
        assert torch.equal(y, want)
        with torch.cuda.graph(graph, stream=s):
            moevie.moevie_checkpoint_store(x, out=ck)
            moevie.moevie_checkpoint_load(ck, out=y)
    new = _rows(300, 1032, torch.bfloat16, 4)
    x.copy_(new)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, moevie.moevie_checkpoint_load(moevie.moevie_checkpoint_store(new)))


def test_no_rows():
    ck = moevie.moevie_checkpoint_store(torch.empty(0, 64, device="cuda"))
    assert moevie.moevie_checkpoint_load(ck).shape == (0, 64)


def test_what_is_refused():
    x = _rows(4, 64, torch.float32, 5)
    for bad in (x.half(), x.t(), x[:, :32], x.cpu()):
        with pytest.raises(ValueError):
            moevie.moevie_checkpoint_store(bad)
    with pytest.raises(moevie.MoevieError) as e:
        moevie.moevie_checkpoint_store(x[:, :12].contiguous())   # d % 8 != 0
    assert e.value.code == 2
    ck = moevie.moevie_checkpoint_store(x)
    with pytest.raises(ValueError):
        moevie.moevie_checkpoint_load(ck, torch.float16)
    with pytest.raises(ValueError):
        moevie.moevie_checkpoint_load(ck, out=torch.empty(3, 64, device="cuda"))


def test_borders_between_codes_of_the_largest_and_smallest_blocks():
    """As above where 1 / amax is subnormal, and at the smallest amax that is kept; and amax / 2, 63.5 codes, of many
    blocks, which is 64."""
    g = torch.Generator()
    g.manual_seed(0)
    top = torch.finfo(torch.float32).max
    some = torch.ldexp(1 + torch.rand(3000, generator=g), torch.tensor(126)) * torch.randint(1, 3, (3000,), generator=g)
    some = some[some < top]
    some = torch.cat([some, torch.tensor([3.3524566e38, 3.35e38, 2.0 ** 127, 2.0 ** 126, 3.4e38, 2.0 ** -110, 1e-33])])
    rows = torch.zeros(len(some), 128)
    rows[:, 0], rows[:, 5], rows[:, 77] = some, some / 2, -some / 2
    ck = _check(rows.cuda())
    assert bool((ck.codes[:, 5] == 64).all()) and bool((ck.codes[:, 77] == -64).all())
    rows = []
    for amax in [2.0 ** 126, 2.0 ** 127, 1.9999999 * 2.0 ** 126, 3.35e38, 3.3524566e38, 3.4e38, 2.0 ** -110, 1e-33]:
        a = torch.tensor(amax, dtype=torch.float32)
        half = ((torch.arange(-127, 127, dtype=torch.float64) + 0.5) * a.double() / 127).float()
        for v in (half, *(torch.nextafter(half, torch.tensor(s)) for s in (float("inf"), float("-inf")))):
            rows += [torch.cat([a.reshape(1), part]) for part in v.split(127)]
    x = torch.stack(rows).cuda()
    assert x.shape[1] == 128
    _check(x)


def test_the_largest_finite_value_comes_back_finite():
    """127 times the nearest float to its 127th part lies beyond it: the scale is the next float below."""
    top = torch.finfo(torch.float32).max
    x = torch.zeros(3, 256, device="cuda")
    x[0, 3], x[1, 200], x[2, 0], x[2, 1], x[2, 2] = top, -top, top, top / 2, -top / 100
    ck = moevie.moevie_checkpoint_store(x)
    got = moevie.moevie_checkpoint_load(ck, torch.float32)
    assert bool(torch.isfinite(got).all())
    assert ck.codes[0, 3] == 127 and ck.codes[1, 200] == -127 and ck.codes[2, 1] == 64 and ck.codes[2, 2] == -1
    scale = ck.scale.repeat_interleave(128, 1).double()
    assert bool(((got.double() - x.double()).abs() <= (0.5 + 127 * 2.0 ** -22) * scale).all())
    below = torch.nextafter(torch.tensor(top), torch.tensor(0.0)).item()
    y = torch.full((1, 128), below, device="cuda")
    _check(y)
