"""GPU: routing by scores where 32 bits end: NaN and infinities in rows whose weights are renormalised, logits and biases
far apart, biases whose sums cancel or overflow; against the plain 64-bit forms.  Tolerances are test_gpu_scored's."""
import numpy as np
import pytest

import scoredref
from test_gpu_scored import DEV, _bias, _check, _f64, _logits, _run

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("T", [40, 6400])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_nan_stays_in_renormalised_softmax_weights(T, bad):
    """A softmax over a NaN or plus infinity is NaN throughout, also where that expert is not selected, may not be, or is
    in another group; the rows beside it are as they were."""
    import torch
    z = _logits(T, 32, 60, "float32")
    rows = [1, 2, 3, T - 1]
    for i, t in enumerate(rows):
        z[t, 5 * i + 2] = float(bad)
    clean = [t for t in range(T) if t not in rows]
    b = _bias(32, 60)
    out = b.clone()
    out[[2, 7, 12, 17]] = -INF
    for bias in (None, b, out):
        for groups, top in ((1, 1), (4, 2)):
            idx, w, _ = _run(z, 4, score="softmax", bias=bias, n_groups=groups, top_groups=top, renorm=True)
            assert torch.isnan(w[rows]).all() and (idx[rows] >= 0).all()
            ri, rw, _ = scoredref.route(_f64(z[clean]), 4, "softmax", None if bias is None else _f64(bias), groups, top, 2, True)
            assert np.array_equal(idx.cpu().numpy()[clean], ri)
            np.testing.assert_allclose(_f64(w)[clean], rw, rtol=2.5e-6, atol=1e-30)


@pytest.mark.parametrize("T", [40, 6400])
def test_selected_logits_far_below_the_largest(T):
    """The expert of the largest logit is ruled out by its bias or its group: the quotients are the selected ones' own."""
    import torch
    z = _logits(T, 16, 61, "float32")
    for t, gap in enumerate((80, 90, 100, 104, 120, 200, 700)):
        z[t, t] += gap
    b = torch.zeros(16, device=DEV)
    b[:8] = -INF
    for bias, groups, top in ((b, 1, 1), (b, 4, 2), (b + torch.arange(16, device=DEV) * 1e-3, 1, 1)):
        for K in (1, 4, 8):
            _check(z, K, "softmax", bias, groups, top, 2, renorm=True, scale=1.5)
            _check(z, K, "softmax", bias, groups, top, 1, renorm=True)


@pytest.mark.parametrize("capped,graph", [(0, 0), (0, 1), (1, 0)])
def test_selected_logits_far_below_the_largest_in_a_decode_context(capped, graph):
    """Expert 0 has a logit of some 150 on every layer and is ruled out by its bias."""
    import torch
    from test_gpu_decode import Stack
    from test_gpu_scored_decode import _context
    from paper_2606_15453_amd import stmoe as S
    from paper_2606_15453_amd import workload as W
    st = Stack(W.CONFIGS["tiny"].scaled(P=8, B=1, T=1))
    cfg = st.cfg
    for l in range(cfg.L):
        x = st.x_dev[0][l][0].float()
        st.wg_dev[l][0] = (x * (150 / (x * x).sum())).to(st.wg_dev[l].dtype)
    bias = torch.zeros((cfg.L, cfg.E), device=DEV)
    bias[:, 0] = -INF
    ctx, pred, keep = _context(st, capped, 0, graph, True)
    ctx.set_routing("softmax", bias)
    y = torch.full((cfg.L, cfg.B, cfg.H), float("nan"), device=DEV)
    ws = torch.empty(S.route_workspace_bytes(cfg.B, cfg.E), dtype=torch.uint8, device=DEV)
    i, w, z = (torch.empty((cfg.B, n), dtype=d, device=DEV) for n, d in
               ((cfg.K, torch.int32), (cfg.K, torch.float32), (cfg.E, torch.float32)))
    ctx.token(0, st.x_dev[0], y, mode=S.MODE_STMOE)
    torch.cuda.synchronize()
    idx, got = ctx.last_routing()
    for l in range(cfg.L):
        S.route_topk(st.x_dev[0][l], st.wg_dev[l], cfg.K, i, w, ws, logits=z)
        assert z[0, 0] > 120
        ri, rw, _ = scoredref.route(_f64(z), cfg.K, "softmax", _f64(bias[l]), renorm=True)
        assert np.array_equal(idx[l], ri)
        np.testing.assert_allclose(got[l], rw, rtol=2.5e-6, atol=1e-30)
    assert torch.isfinite(y).all()
    ctx.close()
    pred.close()


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T", [500, 6500])
def test_groups_by_sums_that_overflow(score, T):
    """Two biases of the type's lowest or largest values: the group's score is beyond 32 bits and still has its place,
    above that of a group without candidates."""
    import torch
    z = _logits(T, 8, 62, "float32")
    low = torch.finfo(torch.float32).min
    for bias, top, K in (([-INF, -INF, low, low, 0, 0, 0, 0], 3, 6), ([low, low, 0.9 * low, low, 0, 0, low, 0.8 * low], 2, 4),
                         ([-INF, low, low, low, -INF, -INF, low, 0], 3, 6), ([-low, -0.9 * low, -low, -low, 0, 0, 0, 0], 1, 2),
                         ([0, 0, -0.7 * low, -0.7 * low, -0.7 * low, -0.8 * low, 1, 1], 2, 3), ([low] * 8, 2, 4)):
        b = torch.tensor(bias, device=DEV)
        for renorm in (False, True):
            _check(z, K, score, b, 4, top, 2, renorm)
        _check(z, K, score, b, 4, top, 1)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("size", [4.0, 64.0, 1000.0, 3e5])
@pytest.mark.parametrize("T", [300, 6500])
def test_groups_by_sums_that_cancel(score, size, T):
    """A group's two choices near +size and -size: rounded to 2^-24 of those in 32 bits, while the sums of different groups
    are nearer than that; seven blocks of eight rows have groups of nearly one score, a part of a rounding to 32 of them
    apart."""
    import torch
    z = _logits(T, 16, 63, "float32")
    k = torch.arange(T, device=DEV)[:, None] // 8 % 8
    z = torch.where(k == 0, z, z * 2.0 ** (k - 22) * size)
    sign = torch.tensor([1.0, -1.0], device=DEV).repeat(8)
    for bias in (size * sign, size * sign + _bias(16, 63, 2.0 ** -10)):
        for top, K in ((4, 8), (3, 2)):
            _check(z, K, score, bias, 8, top, 2)


@pytest.mark.parametrize("T", [9, 6200])
def test_renormalised_sigmoids_of_very_negative_logits(T):
    """Quotients of sigmoids of which some, or all, are below what 32 bits hold."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    z = -20 - 10 * torch.rand((T, 8), generator=torch.Generator(device=DEV).manual_seed(64), device=DEV)
    for t, row in enumerate([[-60, -95], [-60, -88, -89, -105], [-30, -91], [-63.9, -100], [-64.1, -100, -110], [-1, -60],
                             [0, -88, -80], [-200, -210, -260], [5, -70, 90]]):
        z[t] = -INF
        z[t, :len(row)] = torch.tensor(row, device=DEV)
    b = torch.zeros(8, device=DEV)
    for bias in (None, b):
        _check(z, 4, "sigmoid", bias, renorm=True, scale=2.0)
    idx, _, _ = _run(z, 4, score="sigmoid", renorm=True)
    d_w = torch.randn((T, 4), generator=torch.Generator(device=DEV).manual_seed(65), device=DEV)
    out = torch.empty_like(z)
    S.route_scored_backward(z, idx, d_w, out, score="sigmoid", renorm=True)
    ref = scoredref.route_grad(_f64(z), idx.cpu().numpy(), _f64(d_w), "sigmoid", True, 1.0)
    # of an expert's own quotient times a difference of at most twice the largest d_w
    p = scoredref.route(_f64(z), 4, "sigmoid", renorm=True)[1]
    tol = np.zeros_like(ref)
    for t in range(T):
        k = idx[t].cpu().numpy() >= 0
        tol[t, idx[t].cpu().numpy()[k]] = 1e-5 * p[t][k] * np.abs(_f64(d_w[t])).max() + 1e-30
    assert (np.abs(_f64(out) - ref) <= tol).all()
