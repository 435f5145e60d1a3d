"""moevie_balance_loss against its formula in 64 bits; the gradient against automatic differentiation with the
counts held fixed, and against differences."""
import threading

import pytest
import torch

from paper_2608_17402_gb300 import moevie
from tests._block import group_of_rows, runs
from tests._gpu import check_status

pytestmark = pytest.mark.gpu
SENTINEL = 777.0


def loss64(s, idx, rows, G, E, coef, score):
    """Loss and counts of the live rows s (64 bits), rows: the run of each."""
    T, k = idx.shape
    counts = torch.zeros(G, E, dtype=torch.float64, device="cuda")
    ok = (idx >= 0) & (idx < E)
    where = (rows[:, None] * E + idx)[ok]
    counts.view(-1).index_add_(0, where, torch.ones_like(where, dtype=torch.float64))
    lengths = torch.bincount(rows, minlength=G).double().clamp(min=1)[:, None]
    c = coef * E / (k * max(1, T)) * counts / lengths
    empty = (s == float("-inf")).all(1, keepdim=True)
    z = torch.where(empty, torch.zeros_like(s), s)
    p = torch.softmax(z if score == "softmax" else torch.nn.functional.logsigmoid(z), 1)
    return (torch.where(empty, torch.zeros_like(p), p) * c[rows]).sum(), counts.to(torch.int32), c[rows], p


def check(s, idx, score="sigmoid", seg=None, coef=0.03, out=None):
    T, E = s.shape
    G = 1 if seg is None else seg.numel() - 1
    ws = moevie.BalanceWorkspace(T, E, idx.shape[1], G)
    rows = torch.zeros(T, dtype=torch.int64, device="cuda") if seg is None else group_of_rows(T, seg)
    live = rows >= 0
    if out is None:
        out = moevie.BalanceOut.empty(T, E, G)
        out.ds.fill_(SENTINEL)
    moevie.moevie_balance_loss(s, idx, ws, coef, score, seg, out=out)
    check_status(ws)
    z = s.double()[live].requires_grad_()
    loss, counts, c, p = loss64(z, idx.long()[live], rows[live], G, E, coef, score)
    (want,) = torch.autograd.grad(loss, z)
    assert torch.equal(out.counts, counts)
    # a probability is off by a few roundings (2^-21 holds eight), and the loads enter less the even load, whose
    # share of the loss is coef: sums of |p c|
    dev = (c - coef / max(1, int(live.sum()))).abs()
    p = p.detach()
    size = (p * dev).sum(1, keepdim=True)
    # (and the 64-bit form itself, which keeps the even load, loses 2^-53 of it at each of its steps)
    tol = 2.0 ** -19 * p * (dev + size) + 2.0 ** -48 * p * c.abs().sum(1, keepdim=True) + 1e-37
    bad = ~((out.ds.double()[live] - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float(((out.ds.double()[live] - want).abs() / tol).max()))
    loss = float(loss.detach())
    assert abs(float(out.loss) - loss) <= 2.0 ** -20 * (float(size.sum()) + abs(loss))
    assert bool((out.ds[~live] == SENTINEL).all())
    return out


def make(T, E, k, seed=0, skew=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + T + 7 * E)
    s = torch.randn(T, E, generator=g, device="cuda")
    if skew:
        s -= skew * torch.log1p(torch.randperm(E, generator=g, device="cuda").float())
    return s, torch.sort(torch.topk(s, k, dim=1)[1], 1)[0].to(torch.int32)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 1), (3, 4, 2), (5, 5, 3), (512, 16, 2), (77, 17, 4), (1000, 31, 7),
                                   (300, 32, 8), (257, 64, 8), (100, 65, 3), (130, 100, 8), (64, 128, 1), (90, 200, 8),
                                   (70, 201, 4), (2000, 256, 8), (50, 257, 5), (40, 512, 8), (33, 510, 2), (20, 511, 8),
                                   (30, 1024, 8), (9, 1000, 32), (7, 1023, 8), (20000, 64, 8)])
def test_loss_counts_and_gradient(T, E, k, score):
    check(*make(T, E, k, skew=0.5), score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k,G,pad", [(50, 16, 2, 4, (0, 0)), (50, 31, 7, 4, (3, 5)), (1000, 64, 8, 90, (0, 17)),
                                         (300, 128, 8, 1, (10, 20)), (5, 8, 2, 9, (0, 0)), (3000, 256, 8, 33, (0, 0)),
                                         (30, 16, 2, 3, (15, 15)), (40000, 64, 8, 5, (100, 0))])
def test_runs_and_padding(T, E, k, G, pad, score):
    gen = torch.Generator()
    gen.manual_seed(T)
    s, idx = make(T, E, k, skew=0.5)
    seg = runs(T, G, gen, pad)
    dead = group_of_rows(T, seg) < 0
    s[dead] = float("nan")   # padding is not read
    idx[dead] = -5
    check(s, idx, score, seg)


@pytest.mark.parametrize("E", [16, 31, 256])
def test_rows_further_apart_than_wide_and_in_place(E):
    for ld in (E + 1, E + 4, E + 33):
        s, idx = make(200, E, 4)
        big = torch.full((200, ld), SENTINEL, device="cuda")
        big[:, :E] = s
        want = check(s, idx)
        out = moevie.BalanceOut.empty(200, E)
        out.ds = big[:, :E]
        check_in = big[:, :E].clone()
        ws = moevie.BalanceWorkspace(200, E, 4)
        moevie.moevie_balance_loss(big[:, :E], idx, ws, 0.03, out=out)
        assert torch.equal(check_in, s) and torch.equal(out.loss, want.loss)
        # (rows that are not 16 bytes apart are read column by column: the sums' order differs)
        assert bool(((out.ds - want.ds).abs() <= 2.0 ** -18 * want.ds.abs().amax(1, keepdim=True)).all())
        assert bool((big[:, E:] == SENTINEL).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [16, 33])
def test_masked_and_extreme_logits(E, score):
    s, idx = make(64, E, 2)
    s[:, 3] = float("-inf")                       # an expert that is switched off
    s[5] = float("-inf")                          # a row without any
    s[6] = torch.finfo(torch.float32).min         # the type's lowest value everywhere: an even row
    s[7] = s[7] - 200.0                           # sigmoids that vanish in fp32
    s[8, 4:] = torch.finfo(torch.float32).min
    s[9] = s[9] + 90.0                            # sigmoids that are all 1
    s[10, 0], s[10, 1] = 300.0, -300.0
    out = moevie.BalanceOut.empty(64, E)
    ws = moevie.BalanceWorkspace(64, E, 2)
    moevie.moevie_balance_loss(s, idx, ws, 0.03, score, out=out)
    assert bool(torch.isfinite(out.ds).all()) and bool(torch.isfinite(out.loss).all())
    assert not out.ds[5].any() and not out.ds[:, 3][s[:, 3] == float("-inf")].any()
    keep = [t for t in range(64) if t not in (5, 6, 7, 8, 9, 10)]
    finite = s.clone()
    finite[6] = 0.0   # (an even row is any constant, but for the sigmoid's own slope)
    z = finite.double()
    rows = torch.zeros(64, dtype=torch.int64, device="cuda")
    z.requires_grad_()
    loss, _, c, p = loss64(z, idx.long(), rows, 1, E, 0.03, score)
    (want,) = torch.autograd.grad(loss, z)
    dev = (c - 0.03 / 64).abs()
    tol = 2.0 ** -19 * (p * (dev + (p * dev).sum(1, keepdim=True))).detach() + 1e-37
    ok = (out.ds.double() - want).abs() <= tol
    assert bool(ok[keep + [7, 8, 9]].all())
    assert abs(float(out.loss) - float(loss.detach())) <= 2.0 ** -18 * 0.03


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_nan_stays_in_its_row_and_shows_in_the_loss(score):
    s, idx = make(40, 16, 2)
    want = check(s, idx, score)
    s[9, 2] = float("nan")
    got = moevie.moevie_balance_loss(s, idx, moevie.BalanceWorkspace(40, 16, 2), 0.03, score)
    assert bool(torch.isnan(got.loss).all()) and bool(torch.isnan(got.ds[9]).all())
    keep = torch.tensor([t != 9 for t in range(40)])
    assert torch.equal(got.ds[keep], want.ds[keep]) and torch.equal(got.counts, want.counts)


def test_plus_infinity():
    """A softmax has no value there; sigmoids are 1."""
    s, idx = make(40, 16, 2)
    s[3, 5] = float("inf")
    got = moevie.moevie_balance_loss(s, idx, moevie.BalanceWorkspace(40, 16, 2), 0.03, "softmax")
    assert bool(torch.isnan(got.loss).all()) and bool(torch.isnan(got.ds[3]).all())
    assert bool(torch.isfinite(got.ds[[t for t in range(40) if t != 3]]).all())
    got = moevie.moevie_balance_loss(s, idx, moevie.BalanceWorkspace(40, 16, 2), 0.03, "sigmoid")
    s[3, 5] = 80.0   # a sigmoid of 1 in fp32, and its slope below every normal number
    want = moevie.moevie_balance_loss(s, idx, moevie.BalanceWorkspace(40, 16, 2), 0.03, "sigmoid")
    assert torch.equal(got.loss, want.loss) and float(got.ds[3, 5]) == 0
    assert bool(((got.ds - want.ds).abs() <= 1e-30).all())


@pytest.mark.parametrize("E", [8, 16, 31, 64, 256, 300, 1024])
def test_low_rows_among_others(E):
    """Rows of logits far below zero, whose sigmoids have to be taken another way, between ordinary ones: each row's
    gradient is what it is without the others."""
    s, idx = make(97, E, 2)
    shift = torch.tensor([0.0, -12.0, -16.0, -18.0, -30.0, -50.0, -90.0, -1000.0], device="cuda")
    s += shift[torch.arange(97, device="cuda") % 8][:, None]
    check(s, idx)


@pytest.mark.parametrize("E", [8, 33, 256, 1000])
def test_one_logit_at_the_border_of_low_rows(E):
    """Rows of one logit on either side of -17, where the way to take them changes, over others far below it: their
    scores add up to as little as e^-17.  An exponential of x is off by |x| 2^-24 of itself, of 60 at most here (below
    -17 the row's largest logit is taken off first): 2^-18, twice for a probability."""
    s, idx = make(40, E, 2)
    for t, top in enumerate((-16.0, -16.9, -16.9999, -17.0, -17.0001, -17.1, -30.0, -88.0, -100.0)):
        s[t] = top - 43.0
        s[t, (3 * t) % E] = top
    ws = moevie.BalanceWorkspace(40, E, 2)
    out = moevie.moevie_balance_loss(s, idx, ws, 0.03, "sigmoid")
    check_status(ws)
    z = s.double().requires_grad_()
    loss, _, c, p = loss64(z, idx.long(), torch.zeros(40, dtype=torch.int64, device="cuda"), 1, E, 0.03, "sigmoid")
    (want,) = torch.autograd.grad(loss, z)
    p, dev = p.detach(), (c - 0.03 / 40).abs()
    size = (p * dev).sum(1, keepdim=True)
    tol = 2.0 ** -17 * p * (dev + size) + 2.0 ** -48 * p * c.abs().sum(1, keepdim=True) + 1e-37
    assert bool(((out.ds.double() - want).abs() <= tol).all())
    assert abs(float(out.loss) - float(loss.detach())) <= 2.0 ** -17 * (float(size.sum()) + float(loss.detach()))


@pytest.mark.parametrize("T,E,k,G", [(2048, 64, 8, 1), (2049, 64, 8, 1), (4096, 31, 8, 2), (4097, 31, 8, 2), (8192, 16, 8, 4),
                                     (8193, 16, 8, 32)])
def test_both_ways_of_counting(T, E, k, G):
    """On either side of the numbers of ids where the way to count them changes, ids at addresses of 16 bytes and not."""
    s, idx = make(T, E, k, skew=0.5)
    gen = torch.Generator()
    gen.manual_seed(T)
    seg = runs(T, G, gen) if G > 1 else None
    want = check(s, idx, seg=seg)
    apart = torch.empty(T * k + 1, dtype=torch.int32, device="cuda")[1:].view(T, k).copy_(idx)
    got = check(s, apart, seg=seg)
    assert torch.equal(got.loss, want.loss) and torch.equal(got.counts, want.counts) and torch.equal(got.ds, want.ds)


def test_even_loads_have_no_gradient_and_the_loss_coef():
    s, _ = make(64, 16, 2)
    idx = torch.stack([torch.arange(64) % 8, 8 + torch.arange(64) % 8], 1).to(torch.int32).cuda()
    out = check(s, idx, coef=0.25)
    assert not out.ds.any() and float(out.loss) == 0.25


def test_the_same_expert_twice_and_ids_that_are_none():
    s, idx = make(50, 16, 4)
    idx[3] = 7
    check(s, idx)
    idx[4, 1], idx[5, 0] = -1, 16
    ws = moevie.BalanceWorkspace(50, 16, 4)
    out = moevie.moevie_balance_loss(s, idx, ws)
    assert moevie.moevie_get_device_status(ws)[0] == 6
    assert int(out.counts.sum()) == 50 * 4 - 2


def test_runs_that_do_not_ascend_are_a_device_error():
    for bad in ([0, 30, 20, 50], [-3, 10, 20, 50], [0, 10, 20, 51]):
        s, idx = make(50, 16, 2)
        ws = moevie.BalanceWorkspace(50, 16, 2, 3)
        moevie.moevie_balance_loss(s, idx, ws, seg=torch.tensor(bad, dtype=torch.int32, device="cuda"))
        assert moevie.moevie_get_device_status(ws)[0] == 6


def test_gradient_against_differences():
    s, idx = make(6, 12, 3)
    out = check(s, idx)
    z, rows = s.double(), torch.zeros(6, dtype=torch.int64, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    step = torch.randn(6, 12, generator=g, device="cuda", dtype=torch.float64)
    up, down = (loss64(z + h * step, idx.long(), rows, 1, 12, 0.03, "sigmoid")[0] for h in (1e-5, -1e-5))
    slope, along = float(up - down) / 2e-5, float((out.ds.double() * step).sum())
    assert abs(slope - along) <= 1e-5 * float((out.ds.double() * step).abs().sum()) + 1e-10


def test_same_bits_again_on_a_stream_and_in_a_graph():
    s, idx = make(5000, 64, 8, skew=1.0)
    seg = torch.tensor([0, 1000, 1001, 4000, 5000], dtype=torch.int32, device="cuda")
    ws = moevie.BalanceWorkspace(5000, 64, 8, 4)
    want = moevie.moevie_balance_loss(s, idx, ws, seg=seg)
    out = moevie.BalanceOut.empty(5000, 64, 4)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()

    def same():
        return all(torch.equal(x, y) for x, y in ((out.loss, want.loss), (out.counts, want.counts), (out.ds, want.ds)))

    with torch.cuda.stream(st):
        moevie.moevie_balance_loss(s, idx, ws, seg=seg, out=out)
        st.synchronize()
        assert same()
        with torch.cuda.graph(graph, stream=st):
            moevie.moevie_balance_loss(s, idx, ws, seg=seg, out=out)
    for _ in range(3):
        out.ds.zero_()
        out.loss.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert same()


def test_calls_of_two_threads_on_two_streams():
    data = [make(30000, 64, 8, skew=1.0), make(9000, 31, 4, seed=5)]
    spaces = [moevie.BalanceWorkspace(s.shape[0], s.shape[1], idx.shape[1]) for s, idx in data]

    def go(i, stream, out):
        for _ in range(20):
            out[i] = moevie.moevie_balance_loss(*data[i], spaces[i], stream=stream)

    want, got = [None, None], [None, None]
    for i in range(2):
        go(i, None, want)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=go, args=(i, torch.cuda.Stream(), got)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        assert torch.equal(o.loss, w.loss) and torch.equal(o.counts, w.counts) and torch.equal(o.ds, w.ds)


@pytest.mark.parametrize("E", [64, 31])
def test_large_offsets(E):
    """Rows of logits and gradients that lie further apart than 32 bits can count."""
    T, ld = 5, (1 << 29) + 4 if E % 4 == 0 else (1 << 29) + 1
    if torch.cuda.mem_get_info()[0] < 30e9:
        pytest.skip("needs 30 GB")
    s, idx = make(T, E, 4)
    out = moevie.BalanceOut.empty(T, E)
    out.ds = torch.empty(T * ld, device="cuda").view(T, ld)[:, :E]
    far = torch.empty(T * ld, device="cuda").view(T, ld)[:, :E]
    far.copy_(s)
    check(far, idx, out=out)


def test_empty_runs_between_tokens():
    """Thousands of runs, nearly all without a token."""
    G, T = 5000, 60
    ends = torch.zeros(G + 1, dtype=torch.int32)
    ends[1000:], ends[4000:], ends[-1] = 20, 21, T
    s, idx = make(T, 16, 2)
    check(s, idx, seg=ends.cuda())


def test_loss_and_loads_alone_and_no_tokens():
    s, idx = make(300, 31, 4)
    want = check(s, idx)
    got = moevie.moevie_balance_loss(s, idx, moevie.BalanceWorkspace(300, 31, 4), 0.03, grad=False)
    assert got.ds is None and torch.equal(got.loss, want.loss) and torch.equal(got.counts, want.counts)
    none = moevie.moevie_balance_loss(s[:0], idx[:0], moevie.BalanceWorkspace(1, 31, 4))
    assert float(none.loss) == 0 and not none.counts.any()


def test_a_workspace_serves_fewer_tokens_and_runs():
    ws = moevie.BalanceWorkspace(20000, 64, 8, 40)
    for T, G in ((20000, 40), (20000, 1), (9000, 3), (1, 1)):
        s, idx = make(T, 64, 8)
        seg = torch.linspace(0, T, G + 1).to(torch.int32).cuda()
        a = moevie.moevie_balance_loss(s, idx, ws, seg=seg)
        b = moevie.moevie_balance_loss(s, idx, moevie.BalanceWorkspace(T, 64, 8, G), seg=seg)
        assert torch.equal(a.loss, b.loss) and torch.equal(a.ds, b.ds)


def test_what_is_refused():
    s, idx = make(8, 16, 2)
    ws = moevie.BalanceWorkspace(8, 16, 2)
    for bad in ((s.half(), idx), (s.t(), idx), (s, idx.long()), (s, idx[:7]), (s.cpu(), idx)):
        with pytest.raises(ValueError):
            moevie.moevie_balance_loss(*bad, ws)
    with pytest.raises(KeyError):
        moevie.moevie_balance_loss(s, idx, ws, score="relu")
    with pytest.raises(moevie.MoevieError) as e:
        moevie.moevie_balance_loss(s, idx, ws, coef=float("inf"))
    assert e.value.code == 1
    big, ids = make(30000, 16, 2)
    with pytest.raises(moevie.MoevieError) as e:
        moevie.moevie_balance_loss(big, ids, ws)
    assert e.value.code == 3
