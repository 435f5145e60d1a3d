"""moevie_orthogonalize and moevie_muon_update against the formulas evaluated in 64 bits
(X0 = U / |U|_F, X <- a X + (b A + c A^2) X with A = X X^T).

Tolerance of an orthogonalised matrix, 2-norm of the error over 2-norm of the result: each
step rounds X, A and B to fp16 as tensor-core operands (relative rms 2^-11 / sqrt 3 =
2.8e-4).  Fifteen such roundings over five steps add up in quadrature to 1.1e-3, times at
most about 2 for the slope |a + 3 b s^2 + 5 c s^4| of the later steps, so 2.2e-3; the
rounding of the output to bf16 adds 1.7e-3 in quadrature: 2.8e-3.  REL = 4e-3 leaves a
factor 1.4.  Master weights move by lr scale O, so their error is lr scale times that of O
plus a few fp32 roundings."""
import numpy as np
import pytest
import torch

from paper_2608_17402_gb300 import moevie
from tests._gpu import check_status

pytestmark = pytest.mark.gpu

REL = 4e-3
COEF = moevie.NS_COEF


def _ns64(U, coefs):
    """Orthogonalised U [r, c] in 64 bits."""
    X = U.astype(np.float64)
    big = np.abs(X).max()
    if big == 0:
        return X
    X = X / big
    X = X / np.linalg.norm(X)
    flip = X.shape[0] > X.shape[1]
    if flip:
        X = X.T
    for a, b, c in coefs:
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.T if flip else X


def _stack64(U, coefs):
    return np.stack([_ns64(u, coefs) for u in U])


def _f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _rel(got, want):
    return float(np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300))


def _run(U, steps=5, coef=COEF, **kw):
    N, r, c = U.shape if U.dim() == 3 else (1, *U.shape)
    ws = moevie.OrthoWorkspace(N, r, c)
    O = moevie.moevie_orthogonalize(U, ws, coef=coef, steps=steps, **kw)
    check_status(ws)
    return O


def _check(O, U, coefs):
    got, want = _f64(O), _stack64(_f64(U), coefs)
    for e in range(want.shape[0]):   # matrix by matrix: one must not hide another
        assert np.all(np.isfinite(got[e])), e
        assert _rel(got[e], want[e]) <= REL, (e, _rel(got[e], want[e]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,r,c", [(1, 1, 1), (3, 1, 17), (2, 17, 1), (2, 8, 8), (5, 33, 130), (3, 130, 33),
                                   (2, 128, 256), (2, 257, 129), (2, 300, 300), (3, 64, 65), (1, 416, 1664),
                                   (2, 1280, 854), (7, 512, 512), (40, 96, 200), (1, 1100, 1030)])
def test_orthogonalize_full_rank(N, r, c, dtype):
    g = torch.Generator(device="cuda").manual_seed(r * 10007 + c)
    U = torch.randn(N, r, c, generator=g, device="cuda").to(dtype)
    _check(_run(U), U, [COEF] * 5)


@pytest.mark.parametrize("rank", [1, 5, 64])
@pytest.mark.parametrize("r,c", [(384, 200), (200, 384)])
def test_orthogonalize_low_rank(r, c, rank):
    """Few tokens give low-rank gradients: the null directions must stay null."""
    g = torch.Generator(device="cuda").manual_seed(rank)
    U = torch.randn(3, r, rank, generator=g, device="cuda") @ torch.randn(3, rank, c, generator=g, device="cuda")
    _check(_run(U), U, [COEF] * 5)


def test_orthogonalize_scales_zero_and_nonfinite():
    """Each matrix by itself: squares that overflow or vanish in fp32, a zero matrix, and
    matrices holding an infinity or a NaN, which give NaN and leave the others alone."""
    g = torch.Generator(device="cuda").manual_seed(5)
    base = torch.randn(72, 104, generator=g, device="cuda")
    U = torch.stack([base * s for s in (1.0, 1e-30, 1e30, 1e-41, 1e37, 0.0, 1.0, 1.0)])
    U[6, 3, 7] = float("nan")
    U[7, 71, 103] = float("inf")
    O = _run(U)
    # 1e-41 leaves subnormal entries: compare with what they hold
    _check(O[:5], U[:5], [COEF] * 5)
    assert torch.count_nonzero(O[5]) == 0
    assert torch.isnan(O[6]).all() and torch.isnan(O[7]).all()


@pytest.mark.parametrize("steps", [1, 2, 3, 7])
def test_orthogonalize_steps_and_coefficients(steps):
    """Other step counts, a cubic (c = 0: no A^2 product), and coefficients per step."""
    g = torch.Generator(device="cuda").manual_seed(steps)
    U = torch.randn(2, 150, 260, generator=g, device="cuda")
    _check(_run(U, steps=steps), U, [COEF] * steps)
    cubic = (1.5, -0.5, 0.0)
    _check(_run(U, steps=steps, coef=cubic), U, [cubic] * steps)
    mixed = [COEF if i % 2 else cubic for i in range(steps)]
    _check(_run(U, steps=steps, coef=mixed), U, mixed)


def test_orthogonalize_strides():
    """Row and matrix strides of their own for input and output, rows off 16-byte bounds, one
    matrix without a stack, a broadcast stack; nothing outside the output rows is written."""
    g = torch.Generator(device="cuda").manual_seed(1)
    buf = torch.randn(3, 70, 203, generator=g, device="cuda")
    for U in (buf[:, :61, 3:150], buf[:, 5:, :96], buf[1, :, 2:203], buf[:1].expand(4, 70, 203)):
        N = U.shape[0] if U.dim() == 3 else 1
        r, c = U.shape[-2:]
        big = torch.full((N, r + 2, c + 5), 7.0, dtype=torch.bfloat16, device="cuda")
        out = big[:, 1:-1, 3:c + 3]
        out = out[0] if U.dim() == 2 else out
        O = _run(U, out=out)
        assert O.data_ptr() == out.data_ptr()
        _check(out if out.dim() == 3 else out[None], U if U.dim() == 3 else U[None], [COEF] * 5)
        big[:, 1:-1, 3:c + 3] = 7.0
        assert torch.all(big == 7.0)
    t = torch.randn(96, 130, device="cuda").t()
    with pytest.raises(ValueError):
        moevie.moevie_orthogonalize(t, moevie.OrthoWorkspace(1, 130, 96))


def test_orthogonalize_is_deterministic_and_capturable():
    g = torch.Generator(device="cuda").manual_seed(2)
    U = torch.randn(9, 320, 200, generator=g, device="cuda")
    a = _run(U)
    ws = moevie.OrthoWorkspace(9, 320, 200)
    out = torch.empty(U.shape, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()   # a stream other than the tensors' own
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        moevie.moevie_orthogonalize(U, ws, out=out)
    s.synchronize()
    assert torch.equal(a, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moevie.moevie_orthogonalize(U, ws, out=out)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, out)
    check_status(ws)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("N,r,c", [(1, 24, 8), (4, 192, 100), (3, 100, 192), (2, 300, 684), (5, 256, 128)])
def test_muon_update(N, r, c, nesterov):
    g = torch.Generator(device="cuda").manual_seed(N + r + c)

    def rows(std, dtype=torch.float32):
        return moevie.moevie_pad_rows((torch.randn(N, r, c, generator=g, device="cuda") * std).to(dtype))
    W, M, G = rows(r ** -0.5), rows(1e-3), rows(1e-3)
    Wb = moevie.moevie_pad_rows(W.to(torch.bfloat16))
    lr, mu, wd = 0.01, 0.95, 0.1
    scale = 0.2 * max(r, c) ** 0.5
    w, m, gr = _f64(W), _f64(M), _f64(G)
    ws = moevie.OrthoWorkspace(N, r, c)
    for _ in range(2):   # the state of one step feeds the next
        moevie.moevie_muon_update(W, M, G, ws, lr=lr, momentum=mu, weight_decay=wd, nesterov=nesterov, W_bf16=Wb)
        m = mu * m + gr
        O = _stack64(gr + mu * m if nesterov else m, [COEF] * 5)
        w = (1 - lr * wd) * w - lr * scale * O
    check_status(ws)
    assert _rel(_f64(M), m) <= 4 * 2.0 ** -24
    err = np.linalg.norm(_f64(W) - w)
    assert err <= 2 * lr * scale * REL * np.linalg.norm(O) + 8 * 2.0 ** -24 * np.linalg.norm(w), err
    assert torch.equal(Wb, W.to(torch.bfloat16))


def test_muon_update_of_one_matrix_zero_gradients_and_pads():
    """A matrix without a stack; experts without gradient only decay; pad columns of the rows
    are neither read nor written."""
    g = torch.Generator(device="cuda").manual_seed(3)
    W = torch.randn(64, 40, generator=g, device="cuda")
    M, G = torch.zeros_like(W), torch.randn(64, 40, generator=g, device="cuda")
    w, gr = _f64(W), _f64(G)
    ws = moevie.OrthoWorkspace(1, 64, 40)
    moevie.moevie_muon_update(W, M, G, ws, lr=0.5, momentum=0.0, scale=1.0)
    assert _rel(_f64(W), w - 0.5 * _ns64(gr, [COEF] * 5)) <= REL
    assert torch.equal(M, G)

    N, r, c = 3, 20, 13
    bufs = [torch.full((N, r, 16), float("nan"), device="cuda") for _ in range(3)]
    bb = torch.full((N, r, 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    vals = [torch.randn(N, r, c, generator=g, device="cuda") for _ in range(3)]
    vals[1].zero_()       # no momentum yet
    vals[2][1].zero_()    # and no token for expert 1
    for b, v in zip(bufs, vals):
        b[..., :c] = v
    bb[..., :c] = vals[0].to(torch.bfloat16)
    W, M, G = (b[..., :c] for b in bufs)
    ws = moevie.OrthoWorkspace(N, r, c)
    moevie.moevie_muon_update(W, M, G, ws, lr=0.1, weight_decay=0.5, scale=2.0, W_bf16=bb[..., :c])
    check_status(ws)
    want = 0.95 * _f64(vals[0]) - 0.2 * _stack64(_f64(vals[2]) * 1.95, [COEF] * 5)
    assert _rel(_f64(W), want) <= REL
    assert _rel(_f64(W[1]), 0.95 * _f64(vals[0][1])) <= 4 * 2.0 ** -24
    for b in bufs + [bb]:
        assert torch.isnan(b[..., c:]).all() and not torch.isnan(b[..., :c]).any()


def test_empty_stack_is_a_no_op():
    ws = moevie.OrthoWorkspace(1, 16, 16)
    U = torch.zeros(0, 16, 16, device="cuda")
    n0 = moevie.moevie_launch_count()
    assert moevie.moevie_orthogonalize(U, ws).shape == (0, 16, 16)
    assert moevie.moevie_launch_count() == n0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,r,c", [(1, 32, 2048), (3, 20, 1500), (2, 2048, 32), (300, 16, 300), (1, 1500, 5),
                                   (2, 31, 129), (1, 7, 4000), (700, 9, 140), (2, 1, 1030)])
def test_orthogonalize_thin(N, r, c, dtype):
    """At most 32 rows or columns against a long side: one CTA, or several that share it."""
    g = torch.Generator(device="cuda").manual_seed(N + r * 3 + c)
    U = torch.randn(N, r, c, generator=g, device="cuda").to(dtype)
    _check(_run(U), U, [COEF] * 5)
    _check(_run(U, steps=1), U, [COEF])


def test_orthogonalize_thin_nonfinite_zero_and_strides():
    g = torch.Generator(device="cuda").manual_seed(11)
    U = torch.randn(5, 24, 700, generator=g, device="cuda")
    U[1, 2, 3] = float("nan")
    U[2] = 0.0
    U[3, 23, 699] = float("inf")
    O = _run(U)
    _check(O[[0, 4]], U[[0, 4]], [COEF] * 5)
    assert torch.isnan(O[1]).all() and torch.isnan(O[3]).all() and torch.count_nonzero(O[2]) == 0
    wide = torch.randn(5, 26, 713, generator=g, device="cuda")
    out = torch.full((5, 26, 713), 7.0, dtype=torch.bfloat16, device="cuda")
    O = _run(wide[:, 1:25, 5:705], out=out[:, 1:25, 5:705])
    _check(O, wide[:, 1:25, 5:705], [COEF] * 5)
    out[:, 1:25, 5:705] = 7.0
    assert torch.all(out == 7.0)


@pytest.mark.parametrize("N,r,c", [(2, 16, 1200), (3, 700, 30), (400, 8, 72)])
def test_muon_update_thin(N, r, c):
    g = torch.Generator(device="cuda").manual_seed(N + r + c)

    def rows(std, dtype=torch.float32):
        return moevie.moevie_pad_rows((torch.randn(N, r, c, generator=g, device="cuda") * std).to(dtype))
    W, M, G = rows(r ** -0.5), rows(1e-3), rows(1e-3)
    Wb = moevie.moevie_pad_rows(W.to(torch.bfloat16))
    lr, mu, scale = 0.01, 0.9, 0.2 * max(r, c) ** 0.5
    w, m, gr = _f64(W), _f64(M), _f64(G)
    ws = moevie.OrthoWorkspace(N, r, c)
    for nesterov in (True, False):
        moevie.moevie_muon_update(W, M, G, ws, lr=lr, momentum=mu, nesterov=nesterov, W_bf16=Wb)
        m = mu * m + gr
        O = _stack64(gr + mu * m if nesterov else m, [COEF] * 5)
        w = w - lr * scale * O
    check_status(ws)
    assert _rel(_f64(M), m) <= 4 * 2.0 ** -24
    err = np.linalg.norm(_f64(W) - w)
    assert err <= 2 * lr * scale * REL * np.linalg.norm(O) + 8 * 2.0 ** -24 * np.linalg.norm(w), err
    assert torch.equal(Wb, W.to(torch.bfloat16))


@pytest.mark.parametrize("N,r,c,rank", [(2, 100, 512, 7), (1, 2048, 128, 128), (3, 64, 700, 1), (150, 64, 64, 64),
                                        (40, 33, 65, 33), (130, 120, 70, 9), (17, 128, 130, 128)])
def test_orthogonalize_narrow(N, r, c, rank):
    """33 to 128 rows or columns, few matrices and many (a cluster for each, or the tensor
    cores), full rank and low rank; a repeated call gives the same bits."""
    g = torch.Generator(device="cuda").manual_seed(N + r + c + rank)
    if rank < min(r, c):
        U = torch.randn(N, r, rank, generator=g, device="cuda") @ torch.randn(N, rank, c, generator=g, device="cuda")
    else:
        U = torch.randn(N, r, c, generator=g, device="cuda")
    O = _run(U)
    _check(O, U, [COEF] * 5)
    assert torch.equal(_run(U), O)
    cubic = (1.5, -0.5, 0.0)
    _check(_run(U, steps=2, coef=cubic), U, [cubic] * 2)


@pytest.mark.parametrize("N,r,c", [(65, 100, 300), (71, 300, 90), (101, 128, 520), (64, 128, 128), (67, 97, 1000),
                                   (90, 641, 66)])
def test_orthogonalize_stacks_of_narrow_matrices(N, r, c):
    """Stacks whose matrices go through the tiles two by two: odd and even ones, wide and tall;
    rows that are not 16 bytes apart."""
    g = torch.Generator(device="cuda").manual_seed(N + r + c)
    U = torch.randn(N, r, c, generator=g, device="cuda")
    U[3] = 0.0
    U[N - 1] *= 1e-20
    O = _run(U)
    _check(O, U, [COEF] * 5)
    out = torch.full((N, r + 1, c + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(_run(U, out=out[:, :r, 1:c + 1]), O)
    out[:, :r, 1:c + 1] = 7.0
    assert torch.all(out == 7.0)


@pytest.mark.parametrize("N,r,c", [(67, 96, 200), (65, 200, 72)])
def test_muon_update_of_stacks_of_narrow_matrices(N, r, c):
    g = torch.Generator(device="cuda").manual_seed(N + r + c)

    def rows(std, dtype=torch.float32):
        return moevie.moevie_pad_rows((torch.randn(N, r, c, generator=g, device="cuda") * std).to(dtype))
    W, M, G = rows(r ** -0.5), rows(1e-3), rows(1e-3)
    Wb = moevie.moevie_pad_rows(W.to(torch.bfloat16))
    lr, mu, scale = 0.01, 0.9, 0.2 * max(r, c) ** 0.5
    w, m, gr = _f64(W), _f64(M), _f64(G)
    ws = moevie.OrthoWorkspace(N, r, c)
    moevie.moevie_muon_update(W, M, G, ws, lr=lr, momentum=mu, W_bf16=Wb)
    check_status(ws)
    m = mu * m + gr
    O = _stack64(gr + mu * m, [COEF] * 5)
    w = w - lr * scale * O
    for e in (0, 1, N - 2, N - 1):
        err = np.linalg.norm(_f64(W)[e] - w[e])
        assert err <= lr * scale * REL * np.linalg.norm(O[e]) + 8 * 2.0 ** -24 * np.linalg.norm(w[e]), (e, err)
    assert torch.equal(Wb, W.to(torch.bfloat16))
