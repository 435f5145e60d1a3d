"""C ABI of the orthogonalisation and the optimiser step, host side: what is refused, and the
workspace's size.  No call here launches anything."""
import ctypes

import numpy as np
import pytest

from paper_2608_17402_gb300 import moevie

QUINTIC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def lib():
    return moevie.load()


def _codes(lib, coefs, rows, cols, N=2):
    """Status of both entry points for these coefficients, with a workspace of no size: 3 where
    nothing but the workspace is refused."""
    P = ctypes.c_void_p
    fake = P(0x1000)
    co = (ctypes.c_float * (3 * len(coefs)))(*(v for row in coefs for v in row))
    ld = moevie.row_ld(cols)
    return (lib.moevie_orthogonalize(fake, 0, ld, rows * ld, N, rows, cols, co, len(coefs), fake, ld, rows * ld,
                                     fake, 0, None),
            lib.moevie_muon_update(fake, None, fake, fake, N, rows, cols, ld, rows * ld, 0.1, 0.9, 1, 0.0, 1.0, co,
                                   len(coefs), fake, 0, None))


def _largest(coefs):
    """The largest X (but the last), A and b A + c A^2 over singular values in [0, 1], on a grid."""
    top, s = 0.0, 1.0
    for i, (a, b, c) in enumerate(coefs):
        x = np.linspace(0.0, s, 200001)
        t = x * x
        if c != 0:
            top = max(top, t.max())
        top = max(top, np.abs(b * t + c * t * t).max())
        s = np.abs(x * (a + b * t + c * t * t)).max()
        if i + 1 < len(coefs):
            top = max(top, s)
        if top > 1e6:
            break
    return top


@pytest.mark.parametrize("coefs", [
    [QUINTIC] * 5, [QUINTIC] * 32, [(1.5, -0.5, 0.0)] * 32, [(8.0, -12.0, 5.0)], [(0.0, 2.5, -1.5)] * 3,
    [(8.28721, -23.59588, 17.30038), (4.10706, -2.94785, 0.54484), (3.94869, -2.90890, 0.55182)],
    [(100.0, 0.0, 0.0)], [(100.0, 0.0, 0.0)] * 2, [(-59.0, 0.0, 0.0)] * 2, [(7.0, 0.0, 0.0), (1.0, 0.5, 0.01)],
    [(7.0, 0.0, 0.0), (1.0, 0.5, 0.02)], [(1.0, 61.0, 0.0)], [(1.0, -59.0, 0.0)], [(1.0, 100.0, -90.0)],
    [(1.0, 260.0, -259.0)], [(0.0, 0.0, 0.0)] * 2, [(8.0, 0.0, 0.0), (1.0, 0.0, 1e-3)], [(3e38, -3e38, 3e38)] * 32,
    [(200.0, -2000.0, 1801.0), (1.0, 0.0, 0.0)], [(-20.0, 38.75, -19.25)] * 2])
def test_coefficients_have_to_fit_16_bits(lib, coefs):
    """Matrices whose smaller side is above 32 are held in fp16 times 2^10, which ends at 64:
    coefficients that could pass 60 are refused, whatever the stack's size; thin matrices,
    which are held in 32 bits, take any."""
    fits = _largest(np.float32(coefs).astype(np.float64).tolist()) <= 60.0
    for rows, cols, N in ((33, 200, 1), (200, 33, 300), (416, 1664, 2), (1664, 416, 2)):
        want = 3 if fits else 2
        assert _codes(lib, coefs, rows, cols, N) == (want, want), (rows, cols)
    assert _codes(lib, coefs, 32, 4000) == _codes(lib, coefs, 4000, 7) == (3, 3)


@pytest.mark.parametrize("r,c,Ns", [
    (128, 2560, range(1, 400)), (128, 5760, range(1, 200)), (100, 1000, range(1, 1000)), (126, 1316, range(230, 560)),
    (100, 1024, range(400, 480)), (33, 40, range(1, 300)), (416, 1664, range(1, 300)), (1664, 416, range(1, 300)),
    (2560, 128, range(1, 400)), (16, 2048, range(1, 300)), (8192, 8192, range(0, 40)), (129, 300, range(1, 700)),
    (64, 64, range(1, 2000)), (128, 8192, range(50, 200)), (100, 520, list(range(62, 68)) + [65534, 65535])])
def test_workspace_of_a_larger_stack_serves_smaller_ones(lib, r, c, Ns):
    """Stacks of up to N matrices fit a workspace for N."""
    out = ctypes.c_size_t(0)
    prev = 0
    for N in Ns:
        assert lib.moevie_orthogonalize_workspace_size(N, r, c, ctypes.byref(out)) == 0
        assert out.value >= prev, N
        prev = out.value


def test_strides_that_no_tensor_map_holds_are_refused_before_the_momentum_moves(lib):
    """A call that the host refuses has launched nothing, M's update included."""
    P = ctypes.c_void_p
    fake, far = P(0x1000), 1 << 38
    co = (ctypes.c_float * 3)(*QUINTIC)
    n0 = moevie.moevie_launch_count()
    for rows, cols in ((64, 96), (200, 304), (8, 8)):
        def muon(stride, N=2):
            return lib.moevie_muon_update(fake, fake, fake, fake, N, rows, cols, cols, stride, 0.1, 0.9, 1, 0.0, 1.0, co,
                                          1, fake, 1 << 40 if stride >= far else 0, None)

        def ortho(su, so):
            return lib.moevie_orthogonalize(fake, 0, cols, su, 2, rows, cols, co, 1, fake, cols, so, fake,
                                            1 << 40 if max(su, so) >= far else 0, None)
        assert muon(far) == muon(1 << 45) == muon(1 << 60) == 2
        assert ortho(far, rows * cols) == ortho(rows * cols, far) == 2
        assert muon(far - 8) == ortho(far - 8, far - 8) == 3   # (a workspace of no size)
        assert muon(1 << 60, N=0) == 0
    assert moevie.moevie_launch_count() == n0
