"""GPU: 4-bit experts against the plain 64-bit forms.

Tolerances.  Quantising and reading back are exact.  The FFN, relative L2 per
token: three bf16 pieces hold an fp32 value's 24 bits, so with fp32 y what is
left are the fp32 sums of n products, about sqrt(n) 2^-24 of the root sum of
their squares (7e-6 at n = 14336), in a projection, in silu (its slope at most
1.1) times up and in the sum over experts, and the hardware exponential's 2e-6:
2e-5 in all.  With bf16 y the activations (2^-8 at most, independent of each
other) and y itself (2^-8) are rounded: 2^-7.
"""
import numpy as np
import pytest

import mxref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _tol(x_bf16, y_bf16):
    return 2.0 ** -7 if y_bf16 else 2e-5


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


# ------------------------------------------------------------------ quantising
def _quantize(x):
    import torch
    from paper_2606_15453_amd import stmoe as S
    r, c = x.shape
    codes = torch.full((r, (c + 1) // 2), 0xAA, dtype=torch.uint8, device=DEV)
    scales = torch.full((r, (c + 31) // 32), 0xAA, dtype=torch.uint8, device=DEV)
    S.mx_quantize(x, codes, scales)
    out = []
    for dt in (torch.float32, torch.bfloat16):
        y = torch.full((r, c), float("nan"), dtype=dt, device=DEV)
        S.mx_dequantize(codes, scales, y)
        out.append(y)
    return codes.cpu().numpy(), scales.cpu().numpy(), _f64(out[0]), _f64(out[1])


def _check_quantize(x):
    codes, scales, y32, y16 = _quantize(x)
    c, s, v = mxref.mx_quantize(_f64(x))
    assert np.array_equal(scales, s)
    assert np.array_equal(codes, c)
    assert np.array_equal(y32, v, equal_nan=True)
    assert np.array_equal(y16, v, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 8), (7, 100), (64, 512), (33, 1000), (9, 2061),
                                       (1, 8192), (300, 40), (1025, 2)])
def test_quantize_sizes(rows, cols, dtype):
    import torch
    g = torch.Generator(device=DEV).manual_seed(rows * 7919 + cols)
    x = torch.randn((rows, cols), generator=g, device=DEV)
    x *= torch.exp2(torch.randint(-12, 12, (rows, 1), generator=g, device=DEV).float())
    _check_quantize(x.to(getattr(torch, dtype)))


@pytest.mark.parametrize("ld,off", [(64, 0), (65, 0), (72, 0), (72, 3), (80, 8)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_quantize_strided_rows(dtype, ld, off):
    """Rows inside a wider matrix, at any alignment, in and out; what lies between them stays."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    base = torch.randn(20 * ld + off, device=DEV).to(getattr(torch, dtype))
    x = base[off:].view(20, ld)[:, :61]
    _check_quantize(x)
    codes = torch.empty((20, 31), dtype=torch.uint8, device=DEV)
    scales = torch.empty((20, 2), dtype=torch.uint8, device=DEV)
    S.mx_quantize(x, codes, scales)
    out = torch.full_like(base, 7.0)
    y = out[off:].view(20, ld)
    S.mx_dequantize(codes, scales, y[:, :61])
    assert np.array_equal(_f64(y[:, :61]), mxref.mx_quantize(_f64(x))[2])
    assert bool((y[:, 61:] == 7).all()) and bool((out[:off] == 7).all())


def test_quantize_every_border():
    """Every tie of the grid and the fp32 numbers beside it, at every scale, both signs; zeros, subnormal blocks,
    the largest finite values, infinities and NaN."""
    import torch
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, 0, 0.5, 6, 4, 7.5], np.float32)
    near = np.concatenate([ties, np.nextafter(ties, np.float32(9)), np.nextafter(ties, np.float32(-9))])
    rows = []
    for e in range(-149, 126):
        r = np.zeros(96, np.float64)
        r[:39], r[39:78] = near, -near
        r = np.concatenate([np.concatenate([r[i:i + 31], [4.0]]) for i in (0, 31, 62)])     # largest in [4, 8)
        rows.append(np.ldexp(r, e))
    x = np.stack(rows)
    x = np.where(np.abs(x) > np.finfo(np.float32).max, 0, x).astype(np.float32)
    _check_quantize(torch.from_numpy(x).to(DEV))
    x = np.zeros((7, 64), np.float32)
    x[1, 0], x[2, 40], x[3, 5], x[4, 63], x[5, 3] = np.inf, -np.inf, np.nan, -0.0, 3.4e38
    x[6] = 1e-40
    _check_quantize(torch.from_numpy(x).to(DEV))
    _check_quantize(torch.from_numpy(x).to(DEV).to(torch.bfloat16))


def test_dequantize_every_code():
    import torch
    from paper_2606_15453_amd import stmoe as S
    codes = torch.arange(256, dtype=torch.uint8, device=DEV).repeat(256, 1)                      # [256][512 columns]
    scales = torch.arange(256, dtype=torch.uint8, device=DEV).view(256, 1).repeat(1, 16).contiguous()
    want = mxref.mx_values(codes.cpu().numpy(), scales.cpu().numpy(), 512)
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)
    for dt in (torch.float32, torch.bfloat16):
        y = torch.empty((256, 512), dtype=dt, device=DEV)
        S.mx_dequantize(codes, scales, y)
        assert np.array_equal(_f64(y), want, equal_nan=True)


# ------------------------------------------------------------------ experts
class Experts:
    """n random experts: packed blobs and their values in 64 bits."""

    def __init__(self, n, H, I, seed):
        import torch
        from paper_2606_15453_amd import stmoe as S
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.blobs, self.values = [], []
        for _ in range(n):
            mats, vals = [], []
            for r, c in ((I, H), (I, H), (H, I)):
                w = torch.randn((r, c), generator=g, device=DEV) * c ** -0.5
                codes = torch.empty((r, c // 2), dtype=torch.uint8, device=DEV)
                scales = torch.empty((r, (c + 31) // 32), dtype=torch.uint8, device=DEV)
                S.mx_quantize(w, codes, scales)
                mats.append((codes, scales))
                vals.append(mxref.mx_values(codes.cpu().numpy(), scales.cpu().numpy(), c))
            blob = torch.full((S.blob_bytes(H, I, S.MXFP4),), 0xFF, dtype=torch.uint8, device=DEV)
            S.mx_pack_expert(*mats, H, I, blob)
            self.blobs.append(blob)
            self.values.append(vals)
        self.ptrs = torch.tensor([b.data_ptr() for b in self.blobs], dtype=torch.int64, device=DEV)


def _ws(T, K, E, H, I, ns, xd, yd):
    """A workspace full of NaN."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    n = S.ffn_mx_workspace_bytes(T, K, E, H, I, ns, xd, yd)
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)


def _run(ex, E, H, I, x, idx, w, yd, shared=None, ns=0, y=None, ws=None, stream=None):
    import torch
    from paper_2606_15453_amd import stmoe as S
    T, K = idx.shape
    if y is None:
        y = torch.full((T, H), float("nan"), dtype=yd, device=DEV)
    if ws is None:
        ws = _ws(T, K, E, H, I, ns, x.dtype, yd)
    S.expert_ffn_mx(x, idx, w, H, I, E, ex.ptrs, y, ws, shared_ptrs=shared, n_shared=ns, stream=stream)
    return y


def _inputs(T, K, E, H, seed, xd):
    import torch
    rng = np.random.default_rng(seed)
    idx = np.stack([rng.choice(E, K, replace=False) for _ in range(T)]).astype(np.int32) if T else np.zeros((0, K), np.int32)
    w = rng.dirichlet(np.ones(K), size=T).astype(np.float32) if T else np.zeros((0, K), np.float32)
    x = torch.from_numpy(rng.normal(0, 1, (T, H)).astype(np.float32)).to(DEV).to(xd)
    return x, torch.from_numpy(idx).to(DEV), torch.from_numpy(w).to(DEV)


def _err(got, want):
    g, r = _f64(got), np.asarray(want)
    assert np.isfinite(g).all()
    zero = np.linalg.norm(r, axis=1) == 0
    assert not g[zero].any()
    return float((np.linalg.norm(g - r, axis=1)[~zero] / np.linalg.norm(r, axis=1)[~zero]).max()) if (~zero).any() else 0.0


@pytest.mark.parametrize("x_bf16,y_bf16", [(True, False), (True, True), (False, False), (False, True)])
@pytest.mark.parametrize("T,H,I,E,K,ns", [
    (1, 256, 512, 8, 2, 0), (1, 8, 8, 1, 1, 0), (1, 1000, 520, 13, 3, 1), (2, 136, 24, 5, 5, 0), (3, 2048, 768, 16, 8, 0),
    (5, 360, 1408, 9, 2, 2), (8, 512, 640, 40, 4, 0), (15, 264, 264, 7, 3, 1), (16, 1024, 136, 33, 6, 0), (16, 64, 64, 4, 2, 8),
    (17, 256, 256, 6, 2, 0), (37, 1000, 520, 13, 3, 1), (64, 128, 1032, 3, 1, 0), (100, 520, 72, 64, 8, 0), (130, 640, 384, 2, 2, 2),
    (300, 256, 136, 12, 4, 0), (513, 384, 200, 5, 2, 1), (1, 4104, 1544, 3, 2, 0), (9, 4104, 72, 3, 2, 0)])
def test_ffn_parity(T, H, I, E, K, ns, x_bf16, y_bf16):
    import torch
    xd, yd = (torch.bfloat16 if b else torch.float32 for b in (x_bf16, y_bf16))
    ex, sh = Experts(E, H, I, T + H), Experts(ns, H, I, 1)
    x, idx, w = _inputs(T, K, E, H, T * 31 + I, xd)
    y = _run(ex, E, H, I, x, idx, w, yd, shared=sh.ptrs if ns else None, ns=ns)
    want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values, sh.values)
    err = _err(y, want)
    print(f"rel L2 {err:.2e}")
    assert err <= _tol(x_bf16, y_bf16)


@pytest.mark.parametrize("T,H,I,E,K", [(2000, 264, 4104, 20, 2), (8192, 264, 264, 16, 4)])
def test_ffn_prompts_in_large_tiles(T, H, I, E, K):
    """bf16 prompts large enough for tiles of 64 tokens, the down product in parts and whole; a token's bits do not
    depend on the tokens beside it, whichever kind of tile it falls into."""
    import torch
    ex = Experts(E, H, I, T)
    x, idx, w = _inputs(T, K, E, H, 3, torch.bfloat16)
    idx[::50] = -1
    y = _run(ex, E, H, I, x, idx, w, torch.bfloat16)
    want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values)
    assert _err(y, want) <= _tol(True, True)
    x2, idx2, w2 = _inputs(T, K, E, H, 4, torch.bfloat16)
    idx2[:, 0] = 1
    keep = slice(T // 2, T // 2 + 40)
    x2[keep], idx2[keep], w2[keep] = x[keep], idx[keep], w[keep]
    assert torch.equal(_run(ex, E, H, I, x2, idx2, w2, torch.bfloat16)[keep], y[keep])


@pytest.mark.parametrize("H,I", [(4096, 14336), (2048, 1408), (16384, 64), (64, 65536)])
@pytest.mark.parametrize("T", [1, 20])
def test_ffn_large_experts(H, I, T):
    import torch
    ex = Experts(2, H, I, H)
    x, idx, w = _inputs(T, 2, 2, H, I, torch.bfloat16)
    y = _run(ex, 2, H, I, x, idx, w, torch.float32)
    want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values)
    assert _err(y, want) <= _tol(True, False)


@pytest.mark.parametrize("y_bf16", [False, True])
@pytest.mark.parametrize("T,K,E,off", [
    (5, 8, 20, 0), (6, 8, 20, 1), (17, 15, 40, 0), (32, 8, 256, 0), (33, 8, 256, 0), (256, 1, 7, 0), (257, 1, 7, 0), (16, 16, 256, 0), (16, 9, 256, 3), (17, 16, 20, 0), (20, 9, 12, 0), (64, 16, 16, 1),
    (65, 16, 20, 0), (100, 8, 16, 1), (120, 9, 11, 0), (130, 16, 20, 0), (130, 16, 20, 1), (300, 8, 16, 2), (1024, 1, 256, 0),
    (1025, 1, 2, 0), (1100, 12, 64, 0)])
def test_ffn_selections_of_every_width(T, K, E, off, y_bf16):
    """1 to 16 experts per token, in selections at any alignment, around the borders between the ways they are
    sorted; every 7th token repeats its first expert at its end and every 11th selects none."""
    import torch
    H, I = 64, 72
    yd = torch.bfloat16 if y_bf16 else torch.float32
    ex = Experts(E, H, I, T)
    x, sel, w = _inputs(T, K, E, H, K, torch.bfloat16)
    sel[::7, K - 1] = sel[::7, 0]
    sel[::11] = -1
    idx = torch.full((T * K + off,), 2 ** 30, dtype=torch.int32, device=DEV)[off:].view(T, K)
    idx.copy_(sel)
    y = _run(ex, E, H, I, x, idx, w, yd)
    want = mxref.moe_ffn(_f64(x), sel.cpu().numpy(), _f64(w), ex.values)
    assert _err(y, want) <= _tol(True, y_bf16)


@pytest.mark.parametrize("T", [16, 40, 300])
def test_ffn_bf16_results_of_any_size(T):
    """Tokens whose results lie near both ends of bf16's range, whose experts' terms lie 2^40 apart, or that overflow;
    and a row of W_down 2^12 times its neighbours.  Beyond 16 tokens a term below 2^-14 of the largest of its 64 is off
    by 2^-25 of that: 2^-13 of the neighbours' size for each of two terms, and 2^-7 as everywhere."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    H, I, E, K = 264, 136, 4, 2
    ex = Experts(E, H, I, 21)
    x, idx, w = _inputs(T, K, E, H, 6, torch.float32)
    x[0] *= 2.0 ** 60
    x[1] *= 2.0 ** -56
    w[2, 0], w[2, 1] = 1.0, 2.0 ** -40
    x[3] *= 2.0 ** 70
    x = x.to(torch.bfloat16)
    y = _run(ex, E, H, I, x, idx, w, torch.bfloat16)
    want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values)
    rest = [t for t in range(T) if t != 3]
    assert _err(y[rest], want[rest]) <= _tol(True, True)
    assert not bool(y[3].isfinite().all())
    # one row of every expert's W_down, as its scale bytes: row 5, lanes 5, 21, 37 and 53 of the first row block
    h = S.blob_bytes(H, I, S.MXFP4) - 17 * 256
    for e in range(E):
        for lane in (5, 21, 37, 53):
            s = ex.blobs[e][h + 4 * lane:h + 4 * lane + 4]
            s.copy_(torch.where(s > 0, s + 12, s))
        ex.values[e][2][5] *= 4096.0
    keep = [t for t in range(4, T)]
    y = _run(ex, E, H, I, x, idx, w, torch.bfloat16)
    want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values)
    others = [r for r in range(H) if r != 5]
    assert _err(y[keep][:, others], want[keep][:, others]) <= _tol(True, True) + 2 * 2.0 ** -13
    # row 5 itself, a single sum that may cancel: against the sum of its products' magnitudes, of which rounding the
    # activations loses 2^-8, rounding y 2^-8 and rounding the terms 2^-11 (and fp32 the 2e-5 of the other results)
    size = np.zeros(T)
    for t in keep:
        xt = _f64(x[t])
        for e, wk in zip(idx[t].tolist(), _f64(w[t])):
            g, u, d = ex.values[e]
            gx = g @ xt
            size[t] += wk * (np.abs(d[5]) @ np.abs(gx / (1 + np.exp(-gx)) * (u @ xt)))
    off = np.abs(_f64(y)[keep, 5] - want[keep, 5])
    assert (off <= (2.0 ** -7 + 2.0 ** -11 + 2e-5) * size[keep]).all()


@pytest.mark.parametrize("T", [1, 16, 90])
def test_ffn_two_calls_at_once(T):
    """Two streams, a workspace each, both ways of sorting and both result types: the bits of each call alone."""
    import torch
    H, I, E, K = 520, 264, 12, 3
    ex = Experts(E, H, I, 8)
    calls = []
    for i, yd in enumerate((torch.float32, torch.bfloat16)):
        x, idx, w = _inputs(T, K, E, H, i, torch.bfloat16)
        calls.append((x, idx, w, yd, torch.empty((T, H), dtype=yd, device=DEV), _ws(T, K, E, H, I, 0, x.dtype, yd),
                      torch.cuda.Stream(), _run(ex, E, H, I, x, idx, w, yd)))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, idx, w, yd, y, ws, s, _alone in calls:
            _run(ex, E, H, I, x, idx, w, yd, y=y, ws=ws, stream=s)
    torch.cuda.synchronize()
    for *_rest, y, _ws_, _s, alone in calls:
        assert torch.equal(y, alone)


@pytest.mark.parametrize("T", [1, 16, 40, 200])
def test_ffn_in_place(T):
    """y may be x."""
    import torch
    H, I, E, K = 264, 136, 6, 2
    ex = Experts(E, H, I, 3)
    x, idx, w = _inputs(T, K, E, H, 1, torch.bfloat16)
    y = _run(ex, E, H, I, x, idx, w, torch.bfloat16)
    _run(ex, E, H, I, x, idx, w, torch.bfloat16, y=x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("T", [1, 4, 16, 40, 200])
@pytest.mark.parametrize("y_bf16", [False, True])
def test_ffn_odd_selections(T, y_bf16):
    """Rows that select nothing, entries outside the experts, the same expert twice, one expert for all."""
    import torch
    H, I, E, K = 264, 136, 6, 4
    yd = torch.bfloat16 if y_bf16 else torch.float32
    ex = Experts(E, H, I, 3)
    for case in range(4):
        x, idx, w = _inputs(T, K, E, H, case, torch.bfloat16)
        if case == 0:
            idx[::3] = -1
        elif case == 1:
            idx[:, 1], idx[::2, 3] = E, 2 ** 31 - 1
        elif case == 2:
            idx[:, 2] = idx[:, 0]
            idx[::2, 3] = idx[::2, 0]
        else:
            idx[:] = 5
        y = _run(ex, E, H, I, x, idx, w, yd)
        want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values)
        assert _err(y, want) <= _tol(True, y_bf16), case
    idx[:] = -1
    assert not _run(ex, E, H, I, x, idx, w, yd).float().any()


@pytest.mark.parametrize("T", [3, 16, 50, 200])
def test_ffn_bad_tokens_and_experts_stay_alone(T):
    """A token of NaN or infinities, and an expert with a NaN block, change no other token's bits."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    H, I, E, K = 256, 136, 6, 2
    ex = Experts(E, H, I, 5)
    x, idx, w = _inputs(T, K, E, H, 9, torch.bfloat16)
    idx[:] = torch.tensor([0, 1], dtype=torch.int32)
    idx[1] = torch.tensor([2, 1], dtype=torch.int32)
    clean = _run(ex, E, H, I, x, idx, w, torch.float32)
    bad = x.clone()
    bad[0] = float("nan")
    bad[2, 7] = float("inf")
    y = _run(ex, E, H, I, bad, idx, w, torch.float32)
    rest = [t for t in range(T) if t not in (0, 2)]
    assert torch.equal(y[rest], clean[rest])
    assert bool(y[0].isnan().all()) and not bool(y[2].isfinite().all())
    # expert 2 serves token 1 alone: its blob gets a NaN block in every matrix
    blob = ex.blobs[2]
    b = H // 128 * 1024 * ((I + 15) // 16)
    gate_s = 2 * b + 16 * 2 * 1024
    assert S.blob_bytes(H, I, S.MXFP4) == gate_s + 2 * 9 * 256 + 16 * 256
    keep = blob.clone()
    for at in (gate_s, gate_s + 9 * 256, gate_s + 18 * 256):
        blob[at] = 255
    y = _run(ex, E, H, I, x, idx, w, torch.float32)
    blob.copy_(keep)
    rest = [t for t in range(T) if t != 1]
    assert torch.equal(y[rest], clean[rest])
    assert bool(y[1].isnan().any())


def test_ffn_values_beyond_bf16_range_of_fp32_x():
    """fp32 hidden states so large that their bf16 rounding is infinite, and so small that they are subnormal."""
    import torch
    ex = Experts(2, 64, 64, 2)
    x = torch.zeros((3, 64), device=DEV)
    x[0, 0], x[1, 0], x[2, 0] = 3.4028e38, 1e-42, 1.0
    idx = torch.tensor([[0], [1], [1]], dtype=torch.int32, device=DEV)
    w = torch.ones((3, 1), device=DEV)
    y = _run(ex, 2, 64, 64, x, idx, w, torch.float32)
    want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values)
    assert not bool(y[0].isfinite().all())
    assert float(y[1].abs().max()) <= 1e-35
    assert _err(y[2:], want[2:]) <= _tol(False, False)


@pytest.mark.parametrize("x_bf16,y_bf16", [(True, False), (False, False), (False, True)])
@pytest.mark.parametrize("T", [1, 9, 16, 40, 70, 200, 600])
def test_ffn_same_bits_and_independent_tokens(T, x_bf16, y_bf16):
    """The same call twice gives the same bits; beyond a decode step's 16 tokens a token's bits do not depend on the
    tokens beside it as long as the call's size stays (in a step the order of its sums goes by the experts selected)."""
    import torch
    H, I, E, K = 520, 264, 12, 3
    xd, yd = (torch.bfloat16 if b else torch.float32 for b in (x_bf16, y_bf16))
    ex = Experts(E, H, I, 8)
    x, idx, w = _inputs(T, K, E, H, 4, xd)
    out = torch.full((T + 2, H), 5.0, dtype=yd, device=DEV)
    a = _run(ex, E, H, I, x, idx, w, yd, y=out[:T])
    assert bool((out[T:] == 5).all())
    b = _run(ex, E, H, I, x, idx, w, yd)
    assert torch.equal(a, b)
    if T > 1:
        x2, idx2, w2 = _inputs(T, K, E, H, 5, xd)
        keep = slice(T // 2, T // 2 + 9) if T > 32 else slice(T // 2, T // 2 + 1)
        x2[keep], idx2[keep], w2[keep] = x[keep], idx[keep], w[keep]
        c = _run(ex, E, H, I, x2, idx2, w2, yd)
        if T > 16:
            assert torch.equal(c[keep], b[keep])
        else:
            assert _err(c[keep], _f64(b[keep])) <= _tol(x_bf16, y_bf16)


def test_ffn_no_tokens():
    import torch
    ex = Experts(2, 64, 64, 2)
    x, idx, w = _inputs(0, 2, 2, 64, 0, torch.bfloat16)
    assert _run(ex, 2, 64, 64, x, idx, w, torch.float32).shape == (0, 64)


@pytest.mark.parametrize("T", [2, 16, 90])
def test_ffn_other_stream_and_graph(T):
    """On a stream of its own, and captured once and replayed on changing inputs with eager work between."""
    import torch
    H, I, E, K, ns = 256, 264, 10, 3, 1
    ex, sh = Experts(E, H, I, 8), Experts(ns, H, I, 9)
    s = torch.cuda.Stream()
    x, idx, w = _inputs(T, K, E, H, 1, torch.bfloat16)
    ws = _ws(T, K, E, H, I, ns, x.dtype, torch.float32)
    y = torch.empty((T, H), device=DEV)
    torch.cuda.synchronize()
    _run(ex, E, H, I, x, idx, w, torch.float32, shared=sh.ptrs, ns=ns, y=y, ws=ws, stream=s)
    s.synchronize()
    want = mxref.moe_ffn(_f64(x), idx.cpu().numpy(), _f64(w), ex.values, sh.values)
    assert _err(y, want) <= _tol(True, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        _run(ex, E, H, I, x, idx, w, torch.float32, shared=sh.ptrs, ns=ns, y=y, ws=ws, stream=s)
    for seed in range(4):
        x2, idx2, w2 = _inputs(T, K, E, H, 10 + seed, torch.bfloat16)
        x.copy_(x2), idx.copy_(idx2), w.copy_(w2)
        eager = _run(ex, E, H, I, x, idx, w, torch.float32, shared=sh.ptrs, ns=ns)
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager), seed


@pytest.mark.parametrize("T", [2, 90])
def test_ffn_graphs_that_share_a_workspace(T):
    """Two captured calls of different sizes over one workspace, replayed in turn on one stream."""
    import torch
    H, I, E, K = 256, 264, 10, 3
    ex = Experts(E, H, I, 8)
    s = torch.cuda.Stream()
    ws = _ws(T + 40, K, E, H, I, 0, torch.bfloat16, torch.float32)
    graphs = []
    for n in (T, T + 40):
        x, idx, w = _inputs(n, K, E, H, n, torch.bfloat16)
        alone = _run(ex, E, H, I, x, idx, w, torch.float32)
        y = torch.empty((n, H), device=DEV)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            _run(ex, E, H, I, x, idx, w, torch.float32, y=y, ws=ws, stream=s)
        graphs.append((g, y, alone, x, idx, w))
    for i in (0, 1, 1, 0, 1, 0, 0):
        g, y, alone = graphs[i][:3]
        y.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, alone)


def test_ffn_entries_beyond_32_bit_offsets():
    """65536 tokens whose partial rows pass 4 GiB: tokens of both ends and the middle against 64 bits."""
    import torch
    T, H, I, E, K = 65536, 4096, 64, 8, 5
    ex = Experts(E, H, I, 11)
    x, idx, w = _inputs(T, K, E, H, 2, torch.bfloat16)
    y = _run(ex, E, H, I, x, idx, w, torch.bfloat16)
    pick = np.r_[0:40, 32700:32740, T - 40:T]
    want = mxref.moe_ffn(_f64(x[pick]), idx.cpu().numpy()[pick], _f64(w[pick]), ex.values)
    assert _err(y[pick], want) <= _tol(True, True)
    assert bool(y.isfinite().all())


# ------------------------------------------------------------------ the decode context over 4-bit experts
@pytest.mark.parametrize("B,cap", [(1, 0), (3, 0), (16, 0), (1, 3), (4, 5)])
def test_decode_context(B, cap):
    """Whole decode tokens over 4-bit experts, resident and behind a capped cache (host and device decisions), eager
    and as a replayed graph: the selections are moe_route_topk's and every layer's output the FFN's on them."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    Ln, E, K, H, I, ns, tokens = 3, 8, 2, 256, 136, 1, 5
    g = torch.Generator(device=DEV).manual_seed(B)
    router = [(torch.randn((E, H), generator=g, device=DEV)).to(torch.bfloat16) for _ in range(Ln)]
    ex = [Experts(E, H, I, 100 + l) for l in range(Ln)]
    sh = [Experts(ns, H, I, 200 + l) for l in range(Ln)]
    blob = S.blob_bytes(H, I, S.MXFP4)
    rng = np.random.default_rng(B)
    prof = np.stack([np.stack([np.stack([rng.choice(E, K, replace=False) for _ in range(Ln)]) for _ in range(B)])
                     for _ in range(4)]).astype(np.int32)
    pinned = None
    if cap:
        pinned = S.PinnedHost(Ln * E * blob)
        for l in range(Ln):
            for e in range(E):
                pinned.tensor((l * E + e) * blob, blob).copy_(ex[l].blobs[e])
        torch.cuda.synchronize()

    def context(device_policy):
        pred = S.Predictor(Ln, E, K, B)
        pred.profile(prof)
        kw = dict(predictor=pred, shared_ptrs=[b.data_ptr() for l in range(Ln) for b in sh[l].blobs], n_shared=ns)
        keep = [pred]
        if cap:
            n_stage = B * K
            arena, ptr = S.device_workspace(S.cache_arena_bytes(Ln, E, cap, blob, n_stage))
            off = ptr - arena.data_ptr()
            cache = S.ExpertCache(Ln, E, cap, blob, n_stage, arena[off:off + S.cache_arena_bytes(Ln, E, cap, blob, n_stage)],
                                  [pinned.ptr + i * blob for i in range(Ln * E)], torch.cuda.Stream(), torch.cuda.Stream())
            cache.warm(S.warm_sets(prof, E, cap))
            if device_policy:
                cache.set_device_policy(True)
            kw["cache"] = cache
            keep += [cache, arena]
        else:
            kw["resident_ptrs"] = [b.data_ptr() for l in range(Ln) for b in ex[l].blobs]
        ctx = S.DecodeContext(Ln, E, K, B, H, I, S.MXFP4, [r.data_ptr() for r in router], **kw)
        return ctx, keep

    ways = [(False, False)] + ([(True, False), (True, True)] if cap else [(False, True)])
    outs = {}
    for dev_policy, graph in ways:
        ctx, keep = context(dev_policy)
        if graph:
            ctx.set_graph(True)
        outs[dev_policy, graph] = []
        for t in range(tokens):
            gx = torch.Generator(device=DEV).manual_seed(1000 + t)
            xs = torch.randn((Ln, B, H), generator=gx, device=DEV).to(torch.bfloat16)
            ys = torch.full((Ln, B, H), float("nan"), device=DEV)
            ctx.token(t, xs, ys)
            torch.cuda.synchronize()
            idx, w = ctx.last_routing()
            outs[dev_policy, graph].append(ys)
            for l in range(Ln):
                ti = torch.empty((B, K), dtype=torch.int32, device=DEV)
                tw = torch.empty((B, K), device=DEV)
                ws = torch.empty(S.route_workspace_bytes(B, E), dtype=torch.uint8, device=DEV)
                S.route_topk(xs[l], router[l], K, ti, tw, ws)
                assert np.array_equal(ti.cpu().numpy(), idx[l])
                want = mxref.moe_ffn(_f64(xs[l]), idx[l], w[l].astype(np.float64), ex[l].values, sh[l].values)
                assert _err(ys[l], want) <= _tol(True, False)
        ctx.close()
    first = outs[ways[0]]
    for way in ways[1:]:
        assert all(torch.equal(a, b) for a, b in zip(first, outs[way])), way
