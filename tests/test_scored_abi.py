"""Routing by scores without a GPU: refusals before any device work and the plain form the GPU tests compare with."""
import numpy as np
import pytest

import scoredref

S = pytest.importorskip("paper_2606_15453_amd.stmoe")
L = S._lib


def test_route_refusals():
    ok = dict(z=256, T=4, ld=8, E=8, K=2, dt=S.F32, score=S.SIGMOID, bias=None, g=2, tg=1, gt=2, rn=1, scale=1.0, mask=None,
              idx=256, w=256, counts=None)
    for bad in [dict(z=None), dict(idx=None), dict(w=None), dict(T=-1), dict(T=2 ** 26 + 1), dict(ld=7), dict(ld=2 ** 31 + 1),
                dict(E=0), dict(E=257, ld=257), dict(K=0), dict(K=9), dict(K=5), dict(K=17, E=32, ld=32), dict(dt=S.MXFP4),
                dict(dt=9), dict(score=2), dict(score=-1), dict(g=0), dict(g=3), dict(g=9), dict(tg=0), dict(tg=3),
                dict(gt=0), dict(gt=3), dict(scale=float("nan")), dict(scale=float("inf")), dict(z=258),
                dict(z=257, dt=S.BF16)]:
        a = dict(ok, **bad)
        rc = L.moe_route_scored(a["z"], a["T"], a["ld"], a["E"], a["K"], a["dt"], a["score"], a["bias"], a["g"], a["tg"],
                                a["gt"], a["rn"], a["scale"], a["mask"], a["idx"], a["w"], a["counts"], None)
        assert rc == S.EINVAL, bad
        assert L.stmoe_last_error().decode().startswith("moe_route_scored:")
    assert L.moe_route_scored(None, 0, 8, 8, 2, S.F32, 1, None, 1, 1, 2, 0, 1.0, None, None, None, None, None) == S.OK


def test_gradient_and_bias_refusals():
    ok = dict(z=256, T=4, ld=8, E=8, K=2, dt=S.F32, score=S.SIGMOID, rn=0, scale=1.0, idx=256, dw=256, dz=256, ldd=8)
    for bad in [dict(z=None), dict(idx=None), dict(dw=None), dict(dz=None), dict(T=-1), dict(ld=7), dict(ldd=7),
                dict(ldd=2 ** 31 + 1), dict(E=0), dict(K=0), dict(K=9), dict(dt=2), dict(score=3), dict(scale=float("inf")),
                dict(z=258), dict(dz=258)]:
        a = dict(ok, **bad)
        rc = L.moe_route_scored_backward(a["z"], a["T"], a["ld"], a["E"], a["K"], a["dt"], a["score"], a["rn"], a["scale"],
                                         a["idx"], a["dw"], a["dz"], a["ldd"], None)
        assert rc == S.EINVAL, bad
    assert L.moe_route_scored_backward(None, 0, 8, 8, 2, S.F32, 0, 0, 1.0, None, None, None, 8, None) == S.OK
    for args in [(None, 1, 8, 256, 1e-3, 256), (256, 1, 8, None, 1e-3, 256), (256, 1, 8, 256, 1e-3, None),
                 (256, -1, 8, 256, 1e-3, 256), (256, 65536, 8, 256, 1e-3, 256), (256, 1, 0, 256, 1e-3, 256),
                 (256, 1, 257, 256, 1e-3, 256)]:
        assert L.moe_route_bias_step(*args, 0, None) == S.EINVAL
    assert L.moe_route_bias_step(None, 0, 8, None, 1e-3, None, 0, None) == S.OK


def test_binding_refusals():
    """Tensors of the host, other types and shapes never reach the library."""
    import torch
    z, idx, w = torch.zeros(4, 8), torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, 2)
    for f in (lambda: S.route_scored(z, 2, idx, w), lambda: S.route_scored(z[0], 2, idx, w),
              lambda: S.route_scored(z.t(), 2, idx, w), lambda: S.route_scored_backward(z, idx, w, z),
              lambda: S.route_bias_step(idx, w, 1e-3)):
        with pytest.raises((ValueError, RuntimeError)):
            f()
    with pytest.raises(ValueError, match="softmax"):
        S._score("tanh")


def test_plain_form():
    """By hand: a bias changes the choice and not the weight; groups; ties; renormalised and scaled weights."""
    z = np.array([[0.0, 2.0, -1.0, 1.0]])
    s = 1 / (1 + np.exp(-z))
    idx, w, counts = scoredref.route(z, 2, "sigmoid", np.array([1.0, 0, 0, 0]), renorm=True, scale=3.0)
    assert idx.tolist() == [[0, 1]] and counts.tolist() == [1, 1, 0, 0]
    assert np.allclose(w, 3 * s[:, [0, 1]] / s[:, [0, 1]].sum())
    # groups (0, 2) and (-1, 1): by their best one or their sum the first wins; with a bias on -1 the second
    assert scoredref.route(z, 2, "sigmoid", None, 2, 1, 1)[0].tolist() == [[1, 0]]
    assert scoredref.route(z, 2, "sigmoid", np.array([0, 0, 1.0, 0]), 2, 1, 2)[0].tolist() == [[2, 3]]
    assert scoredref.route(np.zeros((1, 4)), 2, "softmax", None, 2, 1, 2)[0].tolist() == [[0, 1]]
    assert scoredref.route(np.full((1, 4), -np.inf), 2, "softmax")[0].tolist() == [[-1, -1]]
    assert scoredref.bias_step([3, 1, 2], np.zeros(3), 0.5).tolist() == [-0.5, 0.5, 0.0]
    e = 1e-6
    for score in ("sigmoid", "softmax"):
        for renorm in (False, True):
            idx, g = np.array([[1, 3]], np.int32), np.array([[0.3, -0.7]])
            f = lambda q: (g * 2 * (lambda p: p / p.sum() if renorm else p)(scoredref.scores(q, score)[0, [1, 3]])).sum()
            d = scoredref.route_grad(z, idx, g, score, renorm, 2.0)
            for j in range(4):
                h = np.eye(4)[j:j + 1] * e
                assert abs((f(z + h) - f(z - h)) / (2 * e) - d[0, j]) < 1e-8
