"""GPU: routing by scores, its gradient and the bias's step against the plain 64-bit forms.

Tolerances.  A choice is compared in 64 bits, so selections are equal.  A weight is a
quotient of exponentials of z or z - max, an argument off by 2^-24 of at most about 20
(1.2e-6 of the exponential); expf's 2^-23, a sum of up to 256 of them, the quotient and
the scale are 2^-20 at most together: 2.5e-6 relative.  A gradient is such a product times
a difference of terms: 1e-5 of the largest term of its row; a bf16 result adds 2^-8 of
itself at most, half a step 2^-9."""
import numpy as np
import pytest

import scoredref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _logits(T, E, seed, dtype, ld=None, off=0):
    import torch
    g = torch.Generator(device=DEV).manual_seed(seed)
    ld = ld or E
    base = torch.randn(T * ld + off, generator=g, device=DEV).to(getattr(torch, dtype)) * 2
    return base[off:].view(T, ld)[:, :E]


def _bias(E, seed, step=1e-3):
    import torch
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-60, 61, (E,), generator=g, device=DEV).float() * step


def _run(z, K, stream=None, **kw):
    import torch
    from paper_2606_15453_amd import stmoe as S
    T, E = z.shape
    idx = torch.full((T, K), 77, dtype=torch.int32, device=DEV)
    w = torch.full((T, K), float("nan"), device=DEV)
    counts = torch.full((E,), 1000, dtype=torch.int32, device=DEV)
    S.route_scored(z, K, idx, w, counts=counts, stream=stream, **kw)
    return idx, w, counts


def _check(z, K, score, bias=None, groups=1, top=None, group_top=2, renorm=False, scale=1.0, mask=None):
    top = groups if top is None else top
    idx, w, counts = _run(z, K, score=score, bias=bias, n_groups=groups, top_groups=top, group_top=group_top, renorm=renorm,
                          scale=scale, mask=mask)
    ri, rw, rc = scoredref.route(_f64(z), K, score, None if bias is None else _f64(bias), groups, top, group_top, renorm,
                                 scale, None if mask is None else mask.cpu().numpy())
    assert np.array_equal(idx.cpu().numpy(), ri)
    np.testing.assert_allclose(_f64(w), rw, rtol=2.5e-6, atol=1e-30)
    assert np.array_equal(counts.cpu().numpy() - 1000, rc)
    return idx, w


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,E,K,groups,top", [(1, 128, 8, 8, 4), (1, 1, 1, 1, 1), (3, 2, 2, 2, 2), (37, 8, 2, 4, 2),
                                              (16, 61, 5, 1, 1), (65, 60, 4, 5, 2), (130, 256, 8, 8, 4), (33, 256, 16, 16, 1),
                                              (50, 64, 6, 64, 9), (20, 48, 16, 3, 2), (9, 192, 7, 4, 3), (70, 16, 16, 2, 2)])
def test_selection(score, dtype, T, E, K, groups, top):
    for seed in range(3):
        z = _logits(T, E, seed, dtype)
        b = _bias(E, seed)
        _check(z, K, score, b, groups, top, 2, renorm=True, scale=2.5)
        _check(z, K, score, b, groups, top, 1, renorm=False)
        _check(z, K, score, None, groups, top, 2, renorm=False, scale=0.5)
        _check(z, K, score, None, groups, top, 1, renorm=True)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,groups,top", [(8, 1, 1), (60, 5, 2), (256, 8, 4)])
def test_ties_go_to_the_lower_index(score, E, groups, top):
    """Equal logits with equal biases, whole rows of them; equal groups."""
    import torch
    z = (_logits(64, E, 1, "float32") / 2).round()
    z[::3] = 0.5
    for b in (None, torch.zeros(E, device=DEV), _bias(E, 2).round(decimals=2)):
        for gt in (1, 2):
            _check(z, 4, score, b, groups, top, gt, renorm=True)
            _check(z.bfloat16(), 4, score, b, groups, top, gt)


def test_near_choices_are_told_apart_in_64_bits():
    """Choices that fp32 rounds to one value or to the wrong order: biases that take back a difference of scores to
    within 1e-9 of each other."""
    import torch
    z = _logits(256, 64, 5, "float32")
    s = 1 / (1 + torch.exp(-z[0].double()))
    b = (0.5 - s).float()                    # row 0: all choices within 3e-8
    z[1::2] = z[0] + 1e-6 * z[1::2]
    for groups, top, gt in [(1, 1, 1), (8, 3, 1), (8, 3, 2)]:
        _check(z, 8, "sigmoid", b, groups, top, gt, renorm=True)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [False, True])
def test_masked_experts_and_rows(score, renorm):
    """Logits and biases of minus infinity, rows and groups with fewer candidates than asked for, rows without any, the
    type's lowest value, masked rows."""
    import torch
    z = _logits(40, 32, 7, "float32")
    b = _bias(32, 7)
    z[0] = -float("inf")
    z[1, 1:] = -float("inf")
    z[2, 5:] = -float("inf")
    z[3, :16] = -float("inf")
    z[4, 2:] = torch.finfo(torch.float32).min
    z[5] = torch.finfo(torch.float32).min
    z[6, ::2] = -float("inf")
    z[7] = -100 - torch.arange(32, device=DEV) / 8
    b[[4, 9, 20]] = -float("inf")
    b[30] = 50.0
    mask = torch.ones(40, dtype=torch.uint8, device=DEV)
    mask[[8, 11, 39]] = 0
    for bias in (b, None):
        for groups, top in ((1, 1), (4, 2), (16, 8)):
            for gt in (1, 2):
                _check(z, 8, score, bias, groups, top, gt, renorm, 1.5, mask)
    _check(z, 8, score, b, 4, 2, 2, renorm, 1.5, mask.bool())


def test_nan_and_infinite_logits():
    import torch
    z = _logits(8, 32, 9, "float32")
    z[1, 3] = float("nan")
    z[2, 7] = float("inf")
    z[3, 4:8] = float("nan")
    clean = [0, 4, 5, 6, 7]
    for bias in (None, _bias(32, 9)):
        idx, w, _ = _run(z, 4, score="sigmoid", bias=bias, n_groups=4, top_groups=2)
        ri, rw, _ = scoredref.route(_f64(z), 4, "sigmoid", None if bias is None else _f64(bias), 4, 2)
        assert np.array_equal(idx.cpu().numpy(), ri)
        np.testing.assert_allclose(_f64(w), rw, rtol=2.5e-6)
        idx, w, _ = _run(z, 4, score="softmax", bias=bias)
        assert torch.isnan(w[1:4]).all() and not torch.isnan(w[clean]).any()
        assert np.array_equal(idx.cpu().numpy()[clean], scoredref.route(
            _f64(z[clean]), 4, "softmax", None if bias is None else _f64(bias))[0])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("E,ld,off", [(61, 64, 3), (64, 65, 1), (128, 131, 2), (256, 260, 4), (200, 201, 0)])
def test_strided_and_unaligned_rows(dtype, E, ld, off):
    _check(_logits(33, E, 11, dtype, ld, off), 6, "sigmoid", _bias(E, 3), renorm=True)
    _check(_logits(33, E, 12, dtype, ld, off), 6, "softmax", _bias(E, 3, 1e-4))


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,E,K,ld", [(1, 8, 2, 8), (37, 60, 4, 64), (130, 256, 8, 257), (65, 128, 16, 128), (5, 1, 1, 3)])
def test_gradient(score, renorm, dtype, T, E, K, ld):
    import torch
    from paper_2606_15453_amd import stmoe as S
    z = _logits(T, E, 13, dtype, ld)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[T // 2] = 0
    idx, _, _ = _run(z, K, score=score, renorm=renorm, mask=mask)
    d_w = torch.randn((T, K), generator=torch.Generator(device=DEV).manual_seed(14), device=DEV)
    out = torch.full((T, ld), float("nan"), dtype=z.dtype, device=DEV)
    S.route_scored_backward(z, idx, d_w, out[:, :E], score=score, renorm=renorm, scale=2.5)
    ref = scoredref.route_grad(_f64(z), idx.cpu().numpy(), _f64(d_w), score, renorm, 2.5)
    big = 2.5 * _f64(d_w.abs().amax(dim=1, keepdim=True))
    tol = 1e-5 * big + (2.0 ** -8 * np.abs(ref) if dtype == "bfloat16" else 0)
    assert (np.abs(_f64(out[:, :E]) - ref) <= tol).all()
    assert torch.isnan(out[:, E:]).all()
    assert not out[T // 2, :E].any() or T == 1 and not mask[0]
    # in place of the logits
    zz = z.clone(memory_format=torch.contiguous_format)
    S.route_scored_backward(zz, idx, d_w, zz, score=score, renorm=renorm, scale=2.5)
    assert torch.equal(zz, out[:, :E])


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(score, renorm):
    """d of sum(w g) along a direction, by central differences of the plain form (64 bits, h = 1e-5: off by 1e-9)."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    z, K = _logits(12, 32, 15, "float32"), 5
    idx, _, _ = _run(z, K, score=score, renorm=renorm)
    d_w = torch.randn((12, K), generator=torch.Generator(device=DEV).manual_seed(16), device=DEV)
    out = torch.empty_like(z)
    S.route_scored_backward(z, idx, d_w, out, score=score, renorm=renorm, scale=1.5)
    z64, e, g = _f64(z), idx.cpu().numpy(), _f64(d_w)

    def f(zz):
        w = np.take_along_axis(scoredref.scores(zz, score), e, 1)
        return (1.5 * (w / w.sum(axis=1, keepdims=True) if renorm else w) * g).sum()

    r = np.random.RandomState(17)
    for _ in range(4):
        d = r.randn(*z64.shape)
        want = (f(z64 + 1e-5 * d) - f(z64 - 1e-5 * d)) / 2e-5
        assert abs((_f64(out) * d).sum() - want) <= 1e-5 * np.abs(_f64(out) * d).sum() + 1e-7


def test_gradient_of_odd_selections():
    """Entries outside the experts, an expert named twice, rows of the lowest value, no entry at all."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    z = _logits(6, 16, 18, "float32")
    z[4] = torch.finfo(torch.float32).min
    z[5] = -90 - torch.arange(16, device=DEV) / 4
    idx = torch.tensor([[3, 3, 1], [-1, 5, -1], [-1, -1, -1], [2, 9, 3], [0, 1, 2], [7, 2, 4]], dtype=torch.int32, device=DEV)
    d_w = torch.randn((6, 3), generator=torch.Generator(device=DEV).manual_seed(19), device=DEV)
    for score in ("sigmoid", "softmax"):
        for renorm in (False, True):
            out = torch.empty_like(z)
            S.route_scored_backward(z, idx, d_w, out, score=score, renorm=renorm)
            ref = scoredref.route_grad(_f64(z), idx.cpu().numpy(), _f64(d_w), score, renorm, 1.0)
            assert (np.abs(_f64(out) - ref) <= 2e-5 * _f64(d_w.abs().amax(dim=1, keepdim=True))).all()
            far = idx.clone()
            far[far < 0] = 16                # beyond the experts: ignored as well
            again = torch.empty_like(z)
            S.route_scored_backward(z, far, d_w, again, score=score, renorm=renorm)
            assert torch.equal(out, again)


@pytest.mark.parametrize("L,E", [(1, 8), (3, 61), (26, 256)])
def test_bias_step(L, E):
    import torch
    from paper_2606_15453_amd import stmoe as S
    r = np.random.RandomState(L)
    c = r.randint(0, 50, (L, E)).astype(np.int32)
    c[0] = 7                                 # all equal: nothing moves
    if L > 1:
        c[1, 0] = 2 ** 31 - 1
    b = r.randn(L, E).astype(np.float32)
    counts, bias = torch.from_numpy(c).to(DEV), torch.from_numpy(b).to(DEV)
    out = torch.full_like(bias, float("nan"))
    S.route_bias_step(counts, bias, 1e-3, out=out)
    want = scoredref.bias_step(c, b.astype(np.float64), 1e-3)
    np.testing.assert_allclose(_f64(out), want, rtol=2.0 ** -23, atol=2.0 ** -34)   # rate and sum, rounded
    assert np.array_equal(out[0].cpu().numpy(), b[0]) and np.array_equal(counts.cpu().numpy(), c)
    S.route_bias_step(counts, bias, 1e-3, reset=True)
    assert torch.equal(bias, out) and not counts.any()
    one = torch.from_numpy(c[L - 1].copy()).to(DEV)
    again = torch.from_numpy(b[L - 1].copy()).to(DEV)
    S.route_bias_step(one, again, 1e-3)
    assert torch.equal(again, out[L - 1])


def test_large_batch_and_repeat():
    """More rows than one pass of the grid; the same bits again; counts of a batch over 2^31 / E rows are not needed."""
    import torch
    z = _logits(20011, 128, 21, "bfloat16")
    b = _bias(128, 21)
    kw = dict(score="sigmoid", bias=b, n_groups=8, top_groups=4, renorm=True)
    first, again = _run(z, 8, **kw), _run(z, 8, **kw)
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    rows = np.random.RandomState(0).choice(20011, 300, replace=False)
    ri, rw, _ = scoredref.route(_f64(z)[rows], 8, "sigmoid", _f64(b), 8, 4, 2, True)
    assert np.array_equal(first[0].cpu().numpy()[rows], ri)
    np.testing.assert_allclose(_f64(first[1])[rows], rw, rtol=2.5e-6)
    assert int(first[2].sum()) - 128 * 1000 == 20011 * 8


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,groups,top", [(7001, 64, 8, 3), (6600, 128, 1, 1), (6200, 64, 32, 9)])
def test_large_batches_with_rows_of_every_kind(score, T, E, groups, top):
    """Beyond the batches of one launch: rows of equal logits (more candidates than the selection in 32 bits takes), near
    ones, NaN, infinities, masked ones, between ordinary ones; their counts are counted once."""
    import torch
    z = _logits(T, E, 50, "float32")
    b = _bias(E, 50, 1e-3 if score == "sigmoid" else 1e-4)
    z[5::97] = 0.25
    z[6::101] = z[6::101].round()
    z[7::103] = z[8] + 1e-6 * z[7::103]
    z[9::211] = -float("inf")
    z[10::223, 3:] = -float("inf")
    z[12::499, 7] = -float("inf")
    z[13::1009, 11] = float("nan") if score == "sigmoid" else 80.0
    z[-1] = z[-2]
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[::41] = 0
    for bias in (b, None, torch.zeros(E, device=DEV)):
        _check(z, 6, score, bias, groups, top, 2, renorm=True, scale=1.5, mask=mask)


def test_streams_and_graphs():
    """On another stream; captured and replayed over new logits between eager work."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    z = [_logits(300, 64, 30 + i, "float32") for i in range(4)]
    b, s = _bias(64, 30), torch.cuda.Stream()
    kw = dict(score="sigmoid", bias=b, n_groups=8, top_groups=3, renorm=True)
    want = [_run(v, 6, **kw) for v in z]
    torch.cuda.synchronize()
    got = _run(z[0], 6, stream=s, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want[0]))
    x, g_w = z[0].clone(), torch.randn((300, 6), device=DEV)
    idx, w = torch.empty((300, 6), dtype=torch.int32, device=DEV), torch.empty((300, 6), device=DEV)
    counts, new, d = torch.zeros(64, dtype=torch.int32, device=DEV), torch.empty(64, device=DEV), torch.empty_like(x)

    def step():
        S.route_scored(x, 6, idx, w, counts=counts, **kw)
        S.route_scored_backward(x, idx, g_w, d, score="sigmoid", renorm=True)
        S.route_bias_step(counts, b, 1e-3, out=new, reset=True)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in (1, 2, 3, 1):
        x.copy_(z[i])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(idx, want[i][0]) and torch.equal(w, want[i][1]) and not counts.any()
        ref = torch.empty_like(d)
        S.route_scored_backward(z[i], idx, g_w, ref, score="sigmoid", renorm=True)
        nb = torch.empty_like(new)
        S.route_bias_step(want[i][2] - 1000, b, 1e-3, out=nb)
        assert torch.equal(d, ref) and torch.equal(new, nb)


def test_offsets_beyond_32_bits():
    """Rows 2^25 elements apart: element offsets beyond 2^32 bytes and 2^31 elements."""
    import torch
    T, E, ld = 72, 64, 1 << 25
    base = torch.zeros((T - 1) * ld + E, dtype=torch.bfloat16, device=DEV)
    z = base.as_strided((T, E), (ld, 1))
    small = _logits(T, E, 40, "bfloat16").contiguous()
    z.copy_(small)
    b = _bias(E, 40)
    got, want = _run(z, 6, score="sigmoid", bias=b), _run(small, 6, score="sigmoid", bias=b)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    from paper_2606_15453_amd import stmoe as S
    d_w, d = torch.randn((T, 6), device=DEV), torch.empty_like(small)
    S.route_scored_backward(small, got[0], d_w, d)
    S.route_scored_backward(z, got[0], d_w, z)
    assert torch.equal(z, d)
