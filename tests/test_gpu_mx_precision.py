"""GPU: bf16 results of the 4-bit expert FFN, every element against a bound that
is derived from the operator's own roundings.

With u = 2^-24 (half a step of fp32), for a token's expert: the sums g and up of
H products are off by (H + 2) u of the sum of the products' magnitudes, silu by
its slope (at most 1.1) of that and by 2e-6 of itself (the hardware's
exponential and reciprocal), their product by 2 u; the activations lose what
their form loses (`act`), and the sums over I products and K experts
(I + K + 4) u of their magnitudes' sum.  y itself is rounded by 2^-8 of itself."""
import numpy as np
import pytest

import mxref
from test_gpu_mx import DEV, _f64, _inputs, _run

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class ScaledExperts:
    """n random experts whose W_down rows are scaled by `rows`: packed blobs and their values in 64 bits."""

    def __init__(self, n, H, I, seed, rows):
        import torch
        from paper_2606_15453_amd import stmoe as S
        g = torch.Generator(device=DEV).manual_seed(seed)
        rows = torch.tensor(rows, dtype=torch.float32, device=DEV)
        self.blobs, self.values = [], []
        for _ in range(n):
            mats, vals = [], []
            for r, c in ((I, H), (I, H), (H, I)):
                w = torch.randn((r, c), generator=g, device=DEV) * c ** -0.5
                if len(mats) == 2:
                    w *= rows[:, None]
                codes = torch.empty((r, c // 2), dtype=torch.uint8, device=DEV)
                scales = torch.empty((r, (c + 31) // 32), dtype=torch.uint8, device=DEV)
                S.mx_quantize(w, codes, scales)
                mats.append((codes, scales))
                vals.append(mxref.mx_values(codes.cpu().numpy(), scales.cpu().numpy(), c))
            blob = torch.empty(S.blob_bytes(H, I, S.MXFP4), dtype=torch.uint8, device=DEV)
            S.mx_pack_expert(*mats, H, I, blob)
            self.blobs.append(blob)
            self.values.append(vals)
        self.ptrs = torch.tensor([b.data_ptr() for b in self.blobs], dtype=torch.int64, device=DEV)


def _want_and_bound(x, idx, w, experts, act, x_bits=0.0):
    """y in 64 bits and how far a bf16 y may be off; x_bits: what x's form loses of it."""
    T, H = x.shape
    I, K = experts[0][0].shape[0], idx.shape[1]
    y, off = np.zeros((T, H)), np.zeros((T, H))
    for e, (gate, up, down) in enumerate(experts):
        hit = idx == e
        rows = np.nonzero(hit.any(axis=1))[0]
        if not len(rows):
            continue
        wt = np.where(hit, w, 0).sum(axis=1)[rows][:, None]
        g, u = x[rows] @ gate.T, x[rows] @ up.T
        e_sum = (H + 2) * U + x_bits
        dg, du = e_sum * (np.abs(x[rows]) @ np.abs(gate).T), e_sum * (np.abs(x[rows]) @ np.abs(up).T)
        s = g / (1 + np.exp(-g))
        h = s * u
        dh = (1.1 * dg + 2e-6 * np.abs(s)) * (np.abs(u) + du) + np.abs(s) * du + (act + 2 * U) * np.abs(h)
        y[rows] += wt * (h @ down.T)
        off[rows] += wt * (((I + K + 4) * U * np.abs(h) + dh) @ np.abs(down).T)
    return y, off + 2.0 ** -8 * (np.abs(y) + off)


def _check(T, H, I, E, K, rows, act, x_bf16=True):
    import torch
    ex = ScaledExperts(E, H, I, 5, rows)
    x, idx, w = _inputs(T, K, E, H, T, torch.bfloat16 if x_bf16 else torch.float32)
    y = _f64(_run(ex, E, H, I, x, idx, w, torch.bfloat16))
    # fp32 x enters in two bf16 pieces: 2^-16 of it
    want, bound = _want_and_bound(_f64(x), idx.cpu().numpy(), _f64(w), ex.values, act, 0.0 if x_bf16 else 2.0 ** -16)
    worst = np.abs(y - want) / bound
    print(f"largest error over its bound {worst.max():.3f}")
    assert (worst <= 1).all()


@pytest.mark.parametrize("T,H,I,E,K", [(4, 264, 136, 4, 2), (16, 264, 136, 4, 2), (40, 264, 136, 4, 2), (300, 264, 136, 4, 2),
                                       (8192, 72, 264, 16, 4)])
def test_small_columns_beside_large_ones(T, H, I, E, K):
    """Columns of y whose W_down rows are 2^-6 to 2^-40 of the others keep their bits (activations in bf16: 2^-8)."""
    rows = [2.0 ** -[0, 0, 6, 14, 20, 26, 40][i % 7] for i in range(H)]
    _check(T, H, I, E, K, rows, act=2.0 ** -8)


@pytest.mark.parametrize("x_bf16", [True, False])
@pytest.mark.parametrize("T,H,I,E,K", [(1, 64, 64, 8, 2), (3, 64, 1544, 6, 4), (8, 64, 64, 8, 2), (9, 64, 64, 8, 2), (16, 64, 64, 8, 2),
                                       (17, 64, 64, 8, 2), (40, 64, 64, 4, 2), (300, 64, 64, 4, 2), (8192, 72, 264, 16, 4)])
def test_bf16_results_are_off_by_their_rounding(T, H, I, E, K, x_bf16):
    """A bf16 y is the fp32 one rounded, but for 2^-16 of the activations (two bf16 pieces)."""
    _check(T, H, I, E, K, [1.0] * H, 2.0 ** -16, x_bf16)
    _check(T, H, I, E, K, [2.0 ** -[0, 0, 6, 14, 20, 26, 40][i % 7] for i in range(H)], 2.0 ** -16, x_bf16)
