"""GPU: the 4-bit expert FFN at the ends of its ranges: infinite results, the widths of hidden states that its
decode kernels divide among waves, offsets beyond 32 bits.  Tolerances as in test_gpu_mx."""
import numpy as np
import pytest

import mxref
from test_gpu_mx import DEV, Experts, _err, _f64, _inputs, _run, _tol

pytestmark = pytest.mark.gpu


def _pack(H, I, gate, up, down):
    """A blob of matrices of the values 0, 1 and -1 (scale 1)."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    mats = []
    for m in (gate, up, down):
        c = torch.where(m == 0, 0, torch.where(m > 0, 2, 10)).to(torch.uint8)
        codes = (c[:, 0::2] | (c[:, 1::2] << 4)).contiguous().to(DEV)
        mats.append((codes, torch.full((m.shape[0], (m.shape[1] + 31) // 32), 127, dtype=torch.uint8, device=DEV)))
    blob = torch.empty(S.blob_bytes(H, I, S.MXFP4), dtype=torch.uint8, device=DEV)
    S.mx_pack_expert(*mats, H, I, blob)
    return blob


@pytest.mark.parametrize("x_bf16,y_bf16", [(True, False), (True, True), (False, False), (False, True)])
@pytest.mark.parametrize("T,E,K", [(1, 4, 2), (5, 4, 2), (16, 4, 2), (17, 4, 2), (40, 4, 2), (300, 4, 2), (8192, 16, 4)])
@pytest.mark.parametrize("H,I", [(72, 264), (136, 328)])
def test_infinite_results(H, I, T, E, K, x_bf16, y_bf16):
    """An infinity among the first hidden states or activations times weights that are not zero there is an infinite
    result, whatever lies behind the last column."""
    import torch

    class Same:
        pass

    xd, yd = (torch.bfloat16 if b else torch.float32 for b in (x_bf16, y_bf16))
    rng = np.random.default_rng(T)
    idx = torch.from_numpy(np.stack([rng.choice(E, K, replace=False) for _ in range(T)]).astype(np.int32)).to(DEV)
    w = torch.full((T, K), 0.5, device=DEV)
    sign = torch.from_numpy(rng.choice([-1, 1], H))
    # x[0] infinite: all gate and up sums are plus infinity, and so is every activation
    gate = torch.zeros((I, H), dtype=torch.int64)
    gate[:, 0] = 1
    down = sign[:, None].expand(H, I)
    # x[0] = 2^65: activation 0 is 2^130, beyond fp32, the others are 0
    one = torch.zeros((I, H), dtype=torch.int64)
    one[0, 0] = 1
    first = torch.zeros((H, I), dtype=torch.int64)
    first[:, 0] = sign
    for x0, mats in ((float("inf"), (gate, gate, down)), (2.0 ** 65, (one, one, first))):
        ex = Same()
        blob = _pack(H, I, *mats)
        ex.ptrs = torch.full((E,), blob.data_ptr(), dtype=torch.int64, device=DEV)
        x = torch.ones((T, H), device=DEV)
        x[:, 0] = x0
        y = _run(ex, E, H, I, x.to(xd), idx, w, yd)
        assert torch.equal(y.float(), (sign * float("inf")).float().to(DEV).expand(T, H)), x0


def _parity(T, H, I, E, K, x_bf16, y_bf16, pick=None, seed=0):
    import torch
    xd, yd = (torch.bfloat16 if b else torch.float32 for b in (x_bf16, y_bf16))
    ex = Experts(E, H, I, T + H)
    x, idx, w = _inputs(T, K, E, H, seed, xd)
    y = _run(ex, E, H, I, x, idx, w, yd)
    pick = np.arange(T) if pick is None else pick
    want = mxref.moe_ffn(_f64(x[pick]), idx.cpu().numpy()[pick], _f64(w[pick]), ex.values)
    assert _err(y[pick], want) <= _tol(x_bf16, y_bf16)
    assert bool(y.isfinite().all())


@pytest.mark.parametrize("y_bf16", [False, True])
@pytest.mark.parametrize("H", [2048, 2056, 3000, 3584, 4096])
@pytest.mark.parametrize("T", [2, 7, 16])
def test_decode_steps_of_wide_hidden_states(T, H, y_bf16):
    """bf16 hidden states of 17 to 32 column tiles (and 16, where the waves are half as many), whose last waves have few
    columns or none: H 2056 leaves three waves of eight without, 3000 two, 3584 one."""
    _parity(T, H, 136, 9, 3, True, y_bf16, seed=H)


@pytest.mark.parametrize("x_bf16,y_bf16", [(True, False), (True, True), (False, False), (False, True)])
@pytest.mark.parametrize("T,H", [(16, 4104), (16, 7168), (7, 5120), (2, 16384)])
def test_decode_steps_of_more_column_tiles(T, H, x_bf16, y_bf16):
    """Hidden states beyond 32 column tiles, and fp32 ones."""
    _parity(T, H, 136, 9, 3, x_bf16, y_bf16, seed=H)


@pytest.mark.parametrize("y_bf16", [False, True])
@pytest.mark.parametrize("H,I", [(4096, 64), (64, 4096)])
def test_terms_and_activations_beyond_32_bit_offsets(H, I, y_bf16):
    """More than 2^31 terms (H) or activations (I), which pass 4 GiB in two bytes each: tokens of both ends and around
    the offsets 2^31 and 2^32."""
    T, E, K = 65536, 9, 9
    n = T * K * max(H, I)
    assert n > 2 ** 31 and 2 * n > 2 ** 32
    edge = [(1 << b) // (K * max(H, I) * size) for b in (31, 32, 33) for size in (1, 2, 4)]
    pick = np.unique(np.concatenate([np.arange(16), np.arange(T - 16, T)] +
                                    [np.arange(max(0, e - 4), min(T, e + 4)) for e in edge]))
    _parity(T, H, I, E, K, True, y_bf16, pick=pick)
