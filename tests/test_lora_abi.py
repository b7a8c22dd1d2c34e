"""Low-rank adapters without a GPU: refusals before any device work, size queries, the plain form."""
import numpy as np
import pytest

import scoredref

S = pytest.importorskip("paper_2606_15453_amd.stmoe")
L = S._lib


def test_plan_sizes_and_refusals():
    for T, n in [(-1, 1), (65537, 1), (4, 0), (4, 4097)]:
        assert S.lora_plan_bytes(T, n) == 0
        assert L.moe_lora_plan(256, T, n, 256, 1 << 30, None) == S.EINVAL
    sizes = [S.lora_plan_bytes(T, 5) for T in (0, 1, 17, 1024, 1025, 65536)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    for a, p, nb in [(None, 256, 1 << 30), (256, None, 1 << 30), (256, 256, 64), (256, 264, 1 << 30), (258, 256, 1 << 30)]:
        assert L.moe_lora_plan(a, 4, 2, p, nb, None) == S.EINVAL
    assert L.moe_lora_plan(None, 0, 2, None, 0, None) == S.OK


def test_workspace_sizes():
    for f in (S.lora_workspace_bytes, S.lora_backward_workspace_bytes):
        for bad in [(-1, 64, 64, 2, 8), (65537, 64, 64, 2, 8), (4, 0, 64, 2, 8), (4, 64, 65537, 2, 8), (4, 64, 64, 0, 8),
                    (4, 64, 64, 4097, 8), (4, 64, 64, 2, 0), (4, 64, 64, 2, 129)]:
            assert f(*bad) == 0
        for Hin, Hout, n, R in [(64, 64, 1, 8), (4096, 4096, 8, 64), (1000, 61, 5, 12), (2048, 61, 64, 128)]:
            sizes = [f(T, Hin, Hout, n, R) for T in list(range(1, 300)) + [511, 512, 1000, 4096, 8191, 8192, 30000, 65536]]
            assert sizes == sorted(sizes) and sizes[0] > 0


def test_lora_refusals():
    ok = dict(x=256, ldx=64, T=4, Hin=64, Hout=32, n=2, R=8, dt=S.BF16, yt=S.F32, plan=256, pb=1 << 20, ap=256, bp=256, ranks=None,
              sc=None, base=256, ldb=32, y=512, ldy=32, v=None, ws=256, nb=1 << 30)
    for bad in [dict(x=None), dict(plan=None), dict(ap=None), dict(bp=None), dict(y=None), dict(ws=None), dict(T=-1),
                dict(T=65537), dict(Hin=0), dict(Hout=0), dict(Hin=65537, ldx=65537), dict(n=0), dict(n=4097), dict(R=0),
                dict(R=129), dict(dt=S.MXFP4), dict(yt=3), dict(ldx=63), dict(ldy=31), dict(ldb=31), dict(ldx=2 ** 31 + 1),
                dict(x=257), dict(y=514), dict(base=257), dict(v=260), dict(plan=264), dict(ws=264), dict(nb=16),
                dict(base=512, ldb=40), dict(pb=300)]:
        a = dict(ok, **bad)
        rc = L.moe_lora(a["x"], a["ldx"], a["T"], a["Hin"], a["Hout"], a["n"], a["R"], a["dt"], a["yt"], a["plan"],
                        a["pb"], a["ap"], a["bp"], a["ranks"], a["sc"], a["base"], a["ldb"], a["y"], a["ldy"], a["v"], a["ws"], a["nb"], None)
        assert rc == S.EINVAL, bad
        assert L.stmoe_last_error().decode().startswith("moe_lora:")
    assert L.moe_lora(None, 64, 0, 64, 32, 2, 8, 1, 0, None, 0, None, None, None, None, None, 0, None, 32, None, None, 0,
                      None) == S.OK


def test_backward_refusals():
    ok = dict(x=256, ldx=64, dy=256, ldy=32, v=256, T=4, Hin=64, Hout=32, n=2, R=8, dt=S.BF16, plan=256, pb=1 << 20, ap=256, bp=256,
              da=256, db=256, base=256, ldb=64, dx=512, ldd=64, ws=256, nb=1 << 30)
    for bad in [dict(x=None), dict(dy=None), dict(v=None), dict(plan=None), dict(ap=None), dict(bp=None), dict(da=None),
                dict(db=None), dict(ws=None), dict(T=0), dict(T=65537), dict(Hin=0), dict(Hout=65537, ldy=65537), dict(n=0),
                dict(R=129), dict(dt=2), dict(ldx=63), dict(ldy=31), dict(ldd=63), dict(ldb=63), dict(x=257), dict(dy=257),
                dict(dx=257), dict(base=257), dict(v=264), dict(plan=264), dict(ws=264), dict(nb=16), dict(base=512, ldb=72),
                dict(dx=256), dict(x=512), dict(pb=300)]:
        a = dict(ok, **bad)
        rc = L.moe_lora_backward(a["x"], a["ldx"], a["dy"], a["ldy"], a["v"], a["T"], a["Hin"], a["Hout"], a["n"], a["R"],
                                 a["dt"], a["plan"], a["pb"], a["ap"], a["bp"], None, None, a["da"], a["db"], a["base"], a["ldb"],
                                 a["dx"], a["ldd"], a["ws"], a["nb"], None)
        assert rc == S.EINVAL, bad
        assert L.stmoe_last_error().decode().startswith("moe_lora_backward:")


def test_binding_refusals():
    import torch
    x, ids, ptrs = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    plan = torch.zeros(S.lora_plan_bytes(4, 2), dtype=torch.uint8)
    for f in (lambda: S.lora_plan(ids, 2, plan), lambda: S.lora(x, plan, ptrs, ptrs, 2, x, plan),
              lambda: S.lora(x[0], plan, ptrs, ptrs, 2, x, plan), lambda: S.lora(x.t(), plan, ptrs, ptrs, 2, x, plan),
              lambda: S.lora_backward(x, x, x, plan, ptrs, ptrs, 2, ptrs, ptrs, plan)):
        with pytest.raises((ValueError, RuntimeError)):
            f()


def test_plain_form():
    """By hand, and the gradient against differences."""
    r = np.random.RandomState(0)
    x, dy, ids = r.randn(5, 3), r.randn(5, 4), np.array([1, -1, 0, 1, 2])
    A, B, s = [r.randn(2, 3), r.randn(1, 3)], [r.randn(2, 4), r.randn(1, 4)], np.array([0.5, 2.0])
    y, v = scoredref.lora(x, ids, A, B, s, np.ones((5, 4)))
    assert np.allclose(y[1], 1) and np.allclose(y[4], 1)           # no adapter: the base
    assert np.allclose(y[0], 1 + 2 * (x[0] @ A[1].T) @ B[1]) and np.allclose(v[2], x[2] @ A[0].T)
    dx, dA, dB = scoredref.lora_grad(x, dy, ids, A, B, s, 0 * x)
    f = lambda x_, A_, B_: (scoredref.lora(x_, ids, A_, B_, s, 0 * dy)[0] * dy).sum()
    h = 1e-5
    p = r.randn(5, 3)
    assert abs((f(x + h * p, A, B) - f(x - h * p, A, B)) / (2 * h) - (dx * p).sum()) < 1e-8
    for k in range(2):
        p, q = r.randn(*A[k].shape), r.randn(*B[k].shape)
        go = lambda e, m, d: [mm + e * d if i == k else mm for i, mm in enumerate(m)]
        assert abs((f(x, go(h, A, p), B) - f(x, go(-h, A, p), B)) / (2 * h) - (dA[k] * p).sum()) < 1e-8
        assert abs((f(x, A, go(h, B, q)) - f(x, A, go(-h, B, q))) / (2 * h) - (dB[k] * q).sum()) < 1e-8
