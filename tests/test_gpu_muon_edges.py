"""moevie_orthogonalize and moevie_muon_update where their coefficients, sizes or stacks are
unusual, against the formulas evaluated in 64 bits.  Tolerances are those of
test_gpu_muon.py unless a test derives its own."""
import numpy as np
import pytest
import torch

from paper_2608_17402_gb300 import moevie
from tests._gpu import check_status
from tests.test_gpu_muon import COEF, REL, _check, _f64, _ns64, _rel, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,r,c", [(101, 128, 520), (71, 300, 90), (2, 200, 300)])
def test_steps_without_a_linear_term(N, r, c):
    """A step with a = 0 takes nothing of X but its products, whose lower parts still count: a
    middle and a last step of that kind, on a workspace that held NaN before it was set up.

    Tolerance: a cubic step has the relative error of one Gram product (two roundings of X,
    2 x 2.8e-4) and passes on three times that of its input; the quintic before it has 5.6e-4,
    the one after it adds as much: 2.8e-3 at the most, 3.3e-3 with the rounding to bf16."""
    g = torch.Generator(device="cuda").manual_seed(N + r)
    U = torch.randn(N, r, c, generator=g, device="cuda")
    cubic = (0.0, 2.5, -1.5)
    for coefs in ([COEF, cubic, COEF], [COEF, cubic]):
        ws = moevie.OrthoWorkspace(N, r, c)
        ws.buf.fill_(255)   # NaN in every floating-point format
        moevie.moevie_workspace_init(ws)
        O = moevie.moevie_orthogonalize(U, ws, coef=coefs, steps=len(coefs))
        check_status(ws)
        _check(O, U, coefs)


def test_entries_near_the_end_of_16_bits():
    """Coefficients under which X reaches 7, A 49 and b A + c A^2 48.5, on matrices whose largest
    singular value is that of a single entry."""
    coefs = [(7.0, 0.0, 0.0), (1.0, 0.5, 0.01)]
    U = torch.zeros(3, 200, 260, device="cuda")
    U[0, 7, 11] = -3.0
    U[1, 199, 259] = 1e-3
    U[2, 0, 0], U[2, 130, 140] = 1.0, 1e-4
    _check(_run(U, steps=2, coef=coefs), U, coefs)
    _check(_run(U[:, :, :20], steps=2, coef=(100.0, 0.0, 0.0)), U[:, :, :20], [(100.0, 0.0, 0.0)] * 2)
    with pytest.raises(moevie.MoevieError) as e:
        _run(U, steps=2, coef=(100.0, 0.0, 0.0))
    assert e.value.code == 2


@pytest.mark.parametrize("N,r,c", [(2, 300, 520), (1, 520, 300)])
def test_last_steps_with_a_large_linear_term(N, r, c):
    """What a step makes of X's lower part in the null directions of U is a times as large as
    it was: with a = 20 and a result of half X, 8e-3 of the result if it is left out.

    Tolerance: X of rank 1 has entries u_i v_j.  Rounding A's, B's and X's by relative 2.8e-4
    (rms) turns the product of B = -19.5 u u^T and X by 2.8e-4 x 19.5 sqrt(3 / m) each, as the
    errors average over m entries: 5.5e-4 for m = 300, 9.5e-4 in quadrature, 1.9e-3 of the
    result.  With the rounding to bf16, 1.7e-3, in quadrature: 2.6e-3."""
    g = torch.Generator(device="cuda").manual_seed(N)
    U = torch.randn(N, r, 1, generator=g, device="cuda") @ torch.randn(N, 1, c, generator=g, device="cuda")
    for coefs in ([(1.5, -0.5, 0.0), (20.0, -38.75, 19.25)],):
        _check(_run(U, steps=2, coef=coefs), U, coefs)
    # one step before the last: its null directions reach the end through a quintic step
    coefs = [(1.5, -0.5, 0.0), (20.0, -38.5, 19.5), (1.5, -0.5, 0.0)]
    _check(_run(U, steps=3, coef=coefs), U, coefs)


def test_matrices_of_a_few_entries():
    """Matrices with at most one entry in a row and a column: every entry is a singular value by
    itself, and no rounding averages.

    Tolerance, entry by entry, with u = 2^-11 the largest relative rounding of an fp16 operand:
    A = x^2 is off by 3u (X twice, its own rounding) and A^2 by 6u, B = b A + c A^2 is rounded
    again and meets a rounded X; in the last two steps up to |a| - 2 and |a| of X's lower part
    are left out; and each step passes on |p'(x)| times the error of its input.  Second-order
    terms: a fifth more per step.  At the end half an ulp of bf16, 2^-9."""
    g = torch.Generator(device="cuda").manual_seed(7)
    N, r, c = 60, 150, 260
    U = torch.zeros(N, r, c, device="cuda")
    for e in range(N):
        k = 1 + e % 6
        i = torch.randperm(r, generator=g, device="cuda")[:k]
        j = torch.randperm(c, generator=g, device="cuda")[:k]
        U[e, i, j] = torch.randn(k, generator=g, device="cuda")
    O = _f64(_run(U))
    u = 2.0 ** -11
    for got, mat in zip(O, _f64(U)):
        want = _ns64(mat, [COEF] * 5)
        assert np.all(got[mat == 0] == 0)
        for q in zip(*np.nonzero(mat)):
            x, err = abs(mat[q]) / np.linalg.norm(mat), 2.0 ** -22
            for it in range(5):
                a, b, cc = COEF
                t = x * x
                B, p, slope = b * t + cc * t * t, abs(x * (a + b * t + cc * t * t)), abs(a + 3 * b * t + 5 * cc * t * t)
                drop = a if it == 4 else a - 2 if it == 3 else 0.0
                err = 1.2 * x * (slope * err + u * (3 * abs(b) * t + 6 * cc * t * t + 2 * abs(B) + drop)) / p
                x = p
            assert abs(got[q] - want[q]) <= (err + 2.0 ** -9) * abs(want[q]), (got[q], want[q], err)


def test_workspace_of_a_larger_stack():
    """A stack that is under way as a whole, in the workspace of one that goes in rounds."""
    g = torch.Generator(device="cuda").manual_seed(8)
    U = torch.randn(144, 128, 2560, generator=g, device="cuda")
    ws = moevie.OrthoWorkspace(145, 128, 2560)
    O = moevie.moevie_orthogonalize(U, ws)
    check_status(ws)
    assert torch.equal(O, _run(U))
    for e in (0, 1, 142, 143):
        _check(O[e:e + 1], U[e:e + 1], [COEF] * 5)


# Stacks that go through the schedule in several groups, a stage apart, whose buffers serve one
# matrix after the other; 256-wide tiles of matrices above 128 rows and columns.  With them, per
# matrix, whether: groups are of unequal size; a mirrored tile, a tile on the diagonal, one that the
# matrix's end trims is 256 wide; the last item of a stack that goes two by two has one matrix.


def _close_on_gpu(O, U, coefs=(COEF,) * 5):
    """The check of every matrix, in 64 bits on the GPU."""
    X = U.double()
    X = X / torch.linalg.vector_norm(X, dim=(1, 2), keepdim=True)
    flip = X.shape[1] > X.shape[2]
    X = X.mT if flip else X
    for a, b, c in coefs:
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    X = X.mT if flip else X
    assert torch.isfinite(O).all()
    rel = torch.linalg.vector_norm(O.double() - X, dim=(1, 2)) / torch.linalg.vector_norm(X, dim=(1, 2))
    assert rel.max().item() <= REL, (int(rel.argmax()), rel.max().item())
    return X


@pytest.mark.parametrize("N,r,c,dtype", [
    (256, 416, 1664, torch.float32), (251, 416, 1664, torch.bfloat16), (97, 1664, 416, torch.float32),
    (301, 128, 2048, torch.float32), (90, 700, 850, torch.float32), (3, 2900, 5000, torch.bfloat16)])
def test_stacks_in_several_groups(N, r, c, dtype):
    g = torch.Generator(device="cuda").manual_seed(N)
    U = torch.randn(N, r, c, generator=g, device="cuda").to(dtype)
    O = _run(U)
    _close_on_gpu(O, U)
    assert torch.equal(_run(U), O)


@pytest.mark.parametrize("N,r,c", [(40, 300, 520), (20, 768, 768), (31, 1280, 854), (40, 290, 1000), (13, 513, 1100),
                                   (80, 257, 256), (100, 180, 250)])
def test_wide_tiles(N, r, c):
    g = torch.Generator(device="cuda").manual_seed(N)
    U = torch.randn(N, r, c, generator=g, device="cuda")
    U[1] = torch.randn(r, 9, generator=g, device="cuda") @ torch.randn(9, c, generator=g, device="cuda")
    U[2] = 0.0
    O = _run(U)
    keep = torch.arange(N, device="cuda") != 2
    _close_on_gpu(O[keep], U[keep])
    assert torch.count_nonzero(O[2]) == 0


@pytest.mark.parametrize("N,r,c,nesterov", [(131, 416, 1664, True), (130, 1664, 416, False), (301, 128, 2048, True),
                                            (31, 1280, 854, True)])
def test_muon_update_of_large_stacks(N, r, c, nesterov):
    g = torch.Generator(device="cuda").manual_seed(N)

    def rows(std):
        return moevie.moevie_pad_rows(torch.randn(N, r, c, generator=g, device="cuda") * std)
    W, M, G = rows(r ** -0.5), rows(1e-3), rows(1e-3)
    Wb = moevie.moevie_pad_rows(W.to(torch.bfloat16))
    lr, mu, wd, scale = 0.02, 0.95, 0.1, 0.2 * max(r, c) ** 0.5
    m = mu * M.double() + G.double()
    u = G.double() + mu * m if nesterov else m
    w = (1 - lr * wd) * W.double()
    ws = moevie.OrthoWorkspace(N, r, c)
    moevie.moevie_muon_update(W, M, G, ws, lr=lr, momentum=mu, weight_decay=wd, nesterov=nesterov, W_bf16=Wb)
    check_status(ws)
    assert (torch.linalg.vector_norm(M.double() - m) <= 4 * 2.0 ** -24 * torch.linalg.vector_norm(m)).item()
    X = u / torch.linalg.vector_norm(u, dim=(1, 2), keepdim=True)
    X = X.mT if r > c else X
    for _ in range(5):
        A = X @ X.mT
        X = COEF[0] * X + (COEF[1] * A + COEF[2] * (A @ A)) @ X
    X = X.mT if r > c else X
    w = w - lr * scale * X
    norm = torch.linalg.vector_norm
    err = norm(W.double() - w, dim=(1, 2))
    most = lr * scale * REL * norm(X, dim=(1, 2)) + 8 * 2.0 ** -24 * norm(w, dim=(1, 2))
    assert (err <= most).all(), (err / most).max().item()
    assert torch.equal(Wb, W.to(torch.bfloat16))


# Tolerance of thin matrices of low or nearly low rank: fp32 throughout, so that null directions hold
# 2^-24 of X, multiplied by a = 3.4445 in every step (3e-5 after five), and within the m x m iteration
# by a^2; a hundred such roundings are 3e-3, with the rounding to bf16, 1.7e-3, 3.5e-3: REL.


@pytest.mark.parametrize("N,r,c,rank", [(16, 25, 95, 1), (5, 8, 53, 1), (3, 114, 16, 1), (1, 30, 35, 3), (36, 312, 4, 1),
                                        (3, 2, 25, 1), (93, 10, 3, 1), (2, 32, 2048, 4), (19, 7, 239, 1),
                                        (13, 314, 26, 3), (2, 2048, 32, 1), (300, 24, 30, 2)])
def test_thin_matrices_of_low_rank(N, r, c, rank):
    g = torch.Generator(device="cuda").manual_seed(N * r + c)
    U = torch.randn(N, r, rank, generator=g, device="cuda") @ torch.randn(N, rank, c, generator=g, device="cuda")
    _check(_run(U), U, [COEF] * 5)
    b = U.to(torch.bfloat16)   # of full rank again, with singular values at its roundings
    _check(_run(b), b, [COEF] * 5)


@pytest.mark.parametrize("N,r,c", [(292, 3, 3), (83, 2, 3), (97, 14, 15), (111, 4, 2), (400, 1, 2)])
def test_small_square_matrices(N, r, c):
    """Many of them, so that some are nearly singular; the update of one step too."""
    g = torch.Generator(device="cuda").manual_seed(N)
    U = torch.randn(N, r, c, generator=g, device="cuda")
    _check(_run(U), U, [COEF] * 5)
    G = moevie.moevie_pad_rows(U)
    W, M = (moevie.moevie_pad_rows(torch.zeros_like(U)) for _ in range(2))
    ws = moevie.OrthoWorkspace(N, r, c)
    moevie.moevie_muon_update(W, M, G, ws, lr=1.0, momentum=0.0, scale=-1.0)
    check_status(ws)
    _check(W, U, [COEF] * 5)


@pytest.mark.parametrize("steps", [6, 7, 10])
@pytest.mark.parametrize("N,r,c,rank", [(16, 25, 95, 1), (2, 32, 2048, 4), (3, 114, 16, 1), (1, 32, 8192, 2), (300, 24, 1500, 3),
                                        (2, 50, 520, 1), (1, 64, 300, 8), (1, 64, 2048, 3), (1, 2048, 60, 5),
                                        (3, 33, 40, 1)])
def test_many_steps_of_low_rank_in_32_bits(N, r, c, rank, steps):
    """Thin and few narrow matrices, in fp32.  X's null directions hold roundings of 2^-24 from every
    step, which the steps after it multiply by a: a^steps 2^-24 sqrt(3) from the first one, 1.4 times
    that from all, several operations a step; 2^-21 a^steps of a result of 0.7 to 1.2 allows for six."""
    g = torch.Generator(device="cuda").manual_seed(N * r + c + steps)
    U = torch.randn(N, r, rank, generator=g, device="cuda") @ torch.randn(N, rank, c, generator=g, device="cuda")
    got, want = _f64(_run(U, steps=steps)), _f64(U)
    for e in range(N):
        w = _ns64(want[e], [COEF] * steps)
        assert _rel(got[e], w) <= REL + 2.0 ** -21 * COEF[0] ** steps, (e, _rel(got[e], w))


@pytest.mark.parametrize("steps", [6, 7])
@pytest.mark.parametrize("N,r,c,rank", [(2, 100, 520, 1), (1, 128, 2048, 3), (1, 2048, 100, 5), (70, 120, 300, 2)])
def test_many_steps_of_low_rank_in_22_bits(N, r, c, rank, steps):
    """The same where X is carried in 22 bits: four times the rounding and half as many operations."""
    g = torch.Generator(device="cuda").manual_seed(N * r + c + steps)
    U = torch.randn(N, r, rank, generator=g, device="cuda") @ torch.randn(N, rank, c, generator=g, device="cuda")
    got, want = _f64(_run(U, steps=steps)), _f64(U)
    for e in range(N):
        w = _ns64(want[e], [COEF] * steps)
        assert _rel(got[e], w) <= REL + 2.0 ** -20 * COEF[0] ** steps, (e, _rel(got[e], w))


@pytest.mark.parametrize("N,r,c", [(16, 25, 95), (2, 32, 2048), (50, 3, 3), (1, 32, 8192), (2, 50, 520), (1, 64, 2048),
                                   (1, 2048, 60), (3, 64, 64)])
def test_many_steps_in_32_bits(N, r, c):
    """Full rank and up to 32 steps: nothing is null, so REL, which has room for the roundings of a
    step (1e-6) times the slopes of those after it."""
    g = torch.Generator(device="cuda").manual_seed(N * r + c)
    U = torch.randn(N, r, c, generator=g, device="cuda")
    for coefs in ([COEF] * 12, [(1.5, -0.5, 0.0)] * 32):
        _check(_run(U, steps=len(coefs), coef=coefs), U, coefs)
