"""GPU: infinities, values at the end of the range and terms that cancel in low-rank adapters against the plain forms in 64
bits: an infinity where the formula has one, NaN where it has NaN, the same numbers elsewhere.

An operand of bf16 is exact in the matrix instruction, the fp32 one (v, u) goes in as pieces: an infinity against a piece
that is 0, or of the other sign than the value, must not show."""
import numpy as np
import pytest

import scoredref
from test_gpu_lora import DEV, Batch, _f64

pytestmark = pytest.mark.gpu
INF = float("inf")


def _same(got, want, what, size=0.0):
    """Infinities and NaN at the same places; numbers within 2^-8 of themselves (half a step of bf16 is 2^-9) and 2^-16 of
    their terms' magnitudes, `size` at most."""
    got, want = _f64(got), np.asarray(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), (what, np.argwhere(np.isnan(got) != np.isnan(want))[:4])
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]) and np.array_equal(np.isinf(got), inf), what
    n = np.isfinite(want)
    assert (np.abs(got[n] - want[n]) <= 2.0 ** -8 * np.abs(want[n]) + 2.0 ** -16 * size).all(), what


def _plain(b):
    with np.errstate(invalid="ignore"):
        return scoredref.lora(_f64(b.x), b.ids, [_f64(m) for m in b.A], [_f64(m) for m in b.B], _f64(b.scales), _f64(b.base))[0]


@pytest.mark.parametrize("T,Hin,Hout,n,R", [(5, 64, 72, 1, 16), (40, 128, 136, 3, 8), (70, 136, 128, 2, 33), (300, 64, 64, 1, 64),
                                            (1100, 72, 64, 2, 128), (20, 61, 33, 2, 12)])
@pytest.mark.parametrize("dtype,ydtype", [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32")])
def test_infinite_adapters_and_rows(dtype, ydtype, T, Hin, Hout, n, R):
    import torch
    b = Batch(T, Hin, Hout, n, R, dtype, ydtype, ids=np.arange(T) % n, seed=70)
    # v and u of one bf16 piece (1 and 4), of several, of pieces of both signs
    for a in range(n):
        b.A[a].zero_()
        b.A[a][:, 0] = 1.0
        b.B[a].zero_()
        b.B[a][:, 0] = 4.0
        b.B[a][R - 1, 5], b.B[a][0, 9], b.B[a][0, 8] = INF, -INF, INF
        b.B[a][R // 2, 8] = INF
    b.scales.fill_(0.5)
    v = torch.empty((T, R), device=DEV)
    for first in (1.0, 1.0 + 2.0 ** -7, -3.0):
        b.x[:, 0] = first
        if T > 2:
            b.x[1, 0] = 0.0                # its own products are NaN
        y = b.forward(v=v)
        _same(y, _plain(b), "y", 6 * R)
    # sums of two terms that need two and three pieces
    if Hin > 1:
        for a in range(n):
            b.A[a][:, 1] = 1.0
        for second in (2.0 ** -9, -2.0 ** -9, 2.0 ** -17, -2.0 ** -20):
            b.x[:, 0], b.x[:, 1] = 1.0, second
            y = b.forward(v=v)
            _same(y, _plain(b), ("y", second), 6 * R)


@pytest.mark.parametrize("T,Hin,Hout,n,R", [(5, 64, 72, 1, 16), (40, 128, 136, 3, 8), (70, 136, 128, 2, 33), (300, 64, 64, 1, 64),
                                            (1500, 72, 64, 1, 128), (2600, 520, 64, 2, 16), (20, 61, 33, 2, 12)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_infinite_rows_and_adapters_of_the_gradient(dtype, T, Hin, Hout, n, R):
    """x reaches dA and dy dB against u and v; A reaches dx against u."""
    import torch
    b = Batch(T, Hin, Hout, n, R, dtype, ids=np.arange(T) % n, seed=71)
    for a in range(n):
        b.A[a].zero_()
        b.B[a].zero_()
        b.B[a][:, 0], b.B[a][:, 1] = 1.0, 1.0
        b.A[a][0, 3], b.A[a][R - 1, 7] = INF, -INF
        b.A[a][:, 10] = INF
    b.scales.fill_(1.0)
    b.dy.zero_()
    b.dy[:, 0], b.dy[:, 1] = 1.0, 2.0 ** -12
    b.x.zero_()
    b.x[0, 2], b.x[T - 1, 5], b.x[T // 2, Hin - 1] = INF, -INF, INF
    v = torch.full((T, R), 1.0 - 2.0 ** -12, device=DEV)
    dx, dA, dB = b.backward(v)
    dbase = _f64(b.dbase)
    with np.errstate(invalid="ignore"):
        rx, rA, _ = scoredref.lora_grad(_f64(b.x), _f64(b.dy), b.ids, [_f64(m) for m in b.A], [_f64(m) for m in b.B],
                                        _f64(b.scales), dbase)
    _same(dx, rx, "dx")
    for a in range(n):
        _same(dA[a], rA[a], "dA")
        rows = np.flatnonzero(b.ids == a)
        _same(dB[a], _f64(v)[rows].T @ _f64(b.dy)[rows], "dB", T)
    # infinities in dy against v of several pieces: u is infinite or NaN and with it dx and dA
    b.dy[0, 4], b.dy[T - 1, Hout - 1] = INF, -INF
    _, dA, dB = b.backward(v)
    for a in range(n):
        rows = np.flatnonzero(b.ids == a)
        with np.errstate(invalid="ignore"):
            _same(dB[a], _f64(v)[rows].T @ _f64(b.dy)[rows], "dB of infinite rows", T)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_sums_at_the_end_of_the_range(dtype):
    """v and u above the largest bf16 number round to an infinity in their first piece and are numbers all the same."""
    import torch
    T, big = 20, 3.395e38
    b = Batch(T, 64, 64, 1, 16, dtype, "float32", ids=np.zeros(T), seed=72)
    b.A[0].zero_()
    b.A[0][:, 0], b.A[0][:, 1] = 2.0 ** 64, 2.0 ** 64
    b.B[0].zero_()
    b.B[0][3, 6] = 0.5
    b.B[0][4, 7] = 2.0 ** -100
    b.x.zero_()
    b.x[:, 0], b.x[:, 1] = 255 * 2.0 ** 56, 127 * 2.0 ** 49     # 2^128 (1 - 2^-8 + 127 2^-15), which rounds up in bf16
    b.scales.fill_(1.0)
    b.base.zero_()
    v = torch.empty((T, 16), device=DEV)
    y = b.forward(v=v)
    assert torch.isfinite(v).all() and (v > big).all()
    want = _f64(v)[0, 0] * np.array([0.5, 2.0 ** -100])
    np.testing.assert_allclose(_f64(y)[:, 6:8], np.tile(want, (T, 1)), rtol=2.0 ** -20)
    assert not y[:, :6].any() and not y[:, 8:].any()
    # dB = v^T dy, one token's own
    b.dy.zero_()
    b.dy[2, 11] = 2.0 ** -100
    _, _, dB = b.backward(v, dx=None)
    np.testing.assert_allclose(_f64(dB[0])[:, 11], want[1], rtol=2.0 ** -20)
    assert not dB[0][:, :11].any() and not dB[0][:, 12:].any()


@pytest.mark.parametrize("T,R", [(3, 2), (40, 16), (200, 24), (70, 64), (150, 100), (1100, 16)])
@pytest.mark.parametrize("ydtype", ["bfloat16", "float32"])
def test_cancelling_terms(ydtype, T, R):
    """v = 1 + 2^-9 + 2^-18, three bf16 pieces, less 1 + 2^-9: exact in 32 bits, and in either type of result; u so."""
    import torch
    b = Batch(T, 64, 64, 1, R, "bfloat16", ydtype, ids=np.zeros(T), seed=73)
    for m in (b.A[0], b.B[0], b.x, b.dy, b.base, b.dbase):
        m.zero_()
    b.scales.fill_(1.0)
    terms = torch.tensor([1.0, 2.0 ** -9, 2.0 ** -18], device=DEV)
    b.x[:, :3], b.dy[:, 5:8] = terms, terms
    b.A[0][0, :3], b.A[0][R - 1, :2] = 1.0, 1.0
    b.B[0][0, 5:8], b.B[0][R - 1, 5:7] = 1.0, 1.0
    b.A[0][0, 20], b.A[0][R - 1, 20] = 1.0, -1.0
    b.B[0][0, 30], b.B[0][R - 1, 30] = 3.0, -3.0
    v = torch.empty((T, R), device=DEV)
    y = b.forward(v=v)
    assert (v[:, 0] == 1 + 2.0 ** -9 + 2.0 ** -18).all()
    assert (y[:, 30] == 3 * 2.0 ** -18).all()
    dx, _, _ = b.backward(v)
    assert (dx[:, 20] == 2.0 ** -18).all()
