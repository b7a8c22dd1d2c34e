"""GPU: low-rank adapters and their gradient against the plain 64-bit forms.

Tolerances.  A sum of N products in fp32 whose terms enter in chains of at most N / 16 + 32
roundings (a matrix instruction adds 4 to 32 products, waves and parts are added at the
end) is off by (N / 16 + 32) 2^-24 of the sum of the products' magnitudes.  v is such a sum
over Hin, y one over the rank of what carries v's error, scaled and added to base in fp32
(2^-22 of both); where y is bf16 v may enter in two bf16 pieces (2^-16 of itself), and y is
off by half a step of bf16, 2^-9 of itself (2^-8 allowed for the sum's own error at a
border).  The gradient so: u over Hout, dx over the rank, dA and dB over the tokens, where
u and v may enter dA and dB in three pieces (2^-23)."""
import numpy as np
import pytest

import scoredref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


class Batch:
    """T tokens, n adapters (of ranks up to R), inputs in `dtype`, base and y in `ydtype`, rows in wider matrices."""

    def __init__(self, T, Hin, Hout, n, R, dtype="bfloat16", ydtype=None, ranks=None, ids=None, seed=0, pad=0, off=0):
        import torch
        from paper_2606_15453_amd import stmoe as S
        self.T, self.Hin, self.Hout, self.n, self.R = T, Hin, Hout, n, R
        self.dt, self.ydt = getattr(torch, dtype), getattr(torch, ydtype or dtype)
        g = torch.Generator(device=DEV).manual_seed(seed)

        def rows(c, dt, scale=1.0):
            flat = (torch.randn(T * (c + pad) + off, generator=g, device=DEV) * scale).to(dt)
            return flat[off:].view(T, c + pad)[:, :c]

        self.rows = rows
        self.x, self.base, self.dy = rows(Hin, self.dt), rows(Hout, self.ydt), rows(Hout, self.dt, 0.1)
        self.dbase = rows(Hin, self.dt)
        r = np.random.RandomState(seed)
        self.ids = r.randint(-1, n + 1, T).astype(np.int32) if ids is None else np.asarray(ids, np.int32)
        self.rank = [R] * n if ranks is None else list(ranks)
        mk = lambda r_, c, s: (torch.randn((r_, c), generator=g, device=DEV) * s).to(self.dt)
        self.A = [mk(k, Hin, Hin ** -0.5) for k in self.rank]
        self.B = [mk(k, Hout, 0.5) for k in self.rank]
        self.scales = torch.rand(n, generator=g, device=DEV) + 0.5
        self.ranks = None if ranks is None else torch.tensor(self.rank, dtype=torch.int32, device=DEV)
        at = lambda ms: torch.tensor([m.data_ptr() if m.numel() else 0 for m in ms], dtype=torch.int64, device=DEV)
        self.ap, self.bp, self.at = at(self.A), at(self.B), at
        self.adapter = torch.from_numpy(self.ids).to(DEV)
        self.plan = torch.full((S.lora_plan_bytes(T, n),), 0xFF, dtype=torch.uint8, device=DEV)
        S.lora_plan(self.adapter, n, self.plan)
        ws = lambda f: torch.full((f(T, Hin, Hout, n, R, self.dt),), 0xFF, dtype=torch.uint8, device=DEV)
        self.ws, self.gws = ws(S.lora_workspace_bytes), ws(S.lora_backward_workspace_bytes)

    def forward(self, base="base", y=None, v=None, stream=None):
        import torch
        from paper_2606_15453_amd import stmoe as S
        y = torch.full((self.T, self.Hout), float("nan"), dtype=self.ydt, device=DEV) if y is None else y
        S.lora(self.x, self.plan, self.ap, self.bp, self.R, y, self.ws, base=self.base if base == "base" else base,
               ranks=self.ranks, scales=self.scales, v=v, stream=stream)
        return y

    def backward(self, v, dx=True, base="base", stream=None):
        import torch
        from paper_2606_15453_amd import stmoe as S
        dA = [torch.full((k, self.Hin), float("nan"), device=DEV) for k in self.rank]
        dB = [torch.full((k, self.Hout), float("nan"), device=DEV) for k in self.rank]
        if dx is True:
            dx = torch.full((self.T, self.Hin), float("nan"), dtype=self.dt, device=DEV)
        S.lora_backward(self.x, self.dy, v, self.plan, self.ap, self.bp, self.R, self.at(dA), self.at(dB), self.gws, dx=dx,
                        base=(self.dbase if base == "base" else base) if dx is not None else None, ranks=self.ranks,
                        scales=self.scales, stream=stream)
        return dx, dA, dB

    def check_forward(self, y, v=None, base=None):
        x, A, B = _f64(self.x), [_f64(m) for m in self.A], [_f64(m) for m in self.B]
        s, b = _f64(self.scales), np.zeros((self.T, self.Hout)) if base is None else _f64(base)
        ref, rv = scoredref.lora(x, self.ids, A, B, s, b)
        bf = "bfloat16" in str(self.ydt)
        tol = np.abs(b) * 4 * EPS
        for t in range(self.T):
            a = self.ids[t]
            if not 0 <= a < self.n or not self.rank[a]:
                continue
            va = np.abs(A[a]) @ np.abs(x[t]) * (self.Hin / 16 + 32) * EPS
            if v is not None:
                got = _f64(v[t])
                assert (np.abs(got[:self.rank[a]] - rv[t]) <= va).all() and not got[self.rank[a]:].any()
            big = np.abs(rv[t]) @ np.abs(B[a])
            tol[t] += s[a] * (va @ np.abs(B[a]) + big * ((self.R / 16 + 36) * EPS + (2.0 ** -16 if bf else 0)))
        if bf:
            tol = tol + 2.0 ** -8 * np.abs(ref)
        err = np.abs(_f64(y) - ref)
        assert (err <= tol).all(), (float((err / np.maximum(tol, 1e-30)).max()), np.argwhere(err > tol)[:4])

    def check_backward(self, dx, dA, dB, base=None):
        x, dy, A, B = _f64(self.x), _f64(self.dy), [_f64(m) for m in self.A], [_f64(m) for m in self.B]
        s, b = _f64(self.scales), np.zeros((self.T, self.Hin)) if base is None else _f64(base)
        rx, rA, rB = scoredref.lora_grad(x, dy, self.ids, A, B, s, b)
        bf, tx = "bfloat16" in str(self.dt), np.abs(b) * 4 * EPS
        for a in range(self.n):
            rows = np.flatnonzero(self.ids == a)
            chain = (len(rows) / 16 + 36) * EPS
            u = s[a] * np.abs(dy[rows]) @ np.abs(B[a]).T                         # magnitudes
            eu = u * (self.Hout / 16 + 34) * EPS
            ev = np.abs(x[rows]) @ np.abs(A[a]).T * (self.Hin / 16 + 32) * EPS
            au = np.abs(s[a] * (dy[rows] @ B[a].T))
            tA = eu.T @ np.abs(x[rows]) + (chain + 2.0 ** -23) * (au.T @ np.abs(x[rows]))
            tB = s[a] * (ev.T @ np.abs(dy[rows]) + (chain + 2.0 ** -22) * (np.abs(x[rows] @ A[a].T).T @ np.abs(dy[rows])))
            assert (np.abs(_f64(dA[a]) - rA[a]) <= tA).all(), ("dA", a)
            assert (np.abs(_f64(dB[a]) - rB[a]) <= tB).all(), ("dB", a)
            tx[rows] += eu @ np.abs(A[a]) + (au @ np.abs(A[a])) * ((self.R / 16 + 34) * EPS + (2.0 ** -16 if bf else 0))
        if dx is not None:
            tx = tx + (2.0 ** -8 * np.abs(rx) if bf else 0)
            assert (np.abs(_f64(dx) - rx) <= tx).all()

    def check(self):
        import torch
        v = torch.full((self.T, self.R), 5.0, device=DEV)
        self.check_forward(self.forward(v=v), v, self.base)
        own = [0 <= a < self.n for a in self.ids]
        assert (v[[not o for o in own]] == 5.0).all()          # rows without an adapter: as they were
        self.check_backward(*self.backward(v), self.dbase)
        return v


SHAPES = [(1, 64, 64, 1, 16), (1, 2048, 2048, 8, 16), (2, 8, 8, 3, 1), (16, 256, 128, 16, 8), (17, 512, 256, 3, 64),
          (37, 1000, 61, 5, 12), (64, 1024, 768, 32, 64), (130, 72, 1032, 2, 33), (300, 520, 1000, 3, 12),
          (33, 264, 24, 40, 128), (600, 384, 640, 2, 100), (5, 1, 1, 2, 3), (50, 31, 257, 4, 20), (2500, 136, 72, 2, 40), (1300, 520, 264, 1, 16),
          (2300, 64, 88, 1, 70), (700, 61, 33, 1, 5),
          (20, 2048, 61, 3, 12), (20, 1027, 64, 3, 8), (20, 61, 2048, 2, 8), (3, 8192, 4096, 2, 16)]


@pytest.mark.parametrize("dtype,ydtype", [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32"),
                                          ("float32", "bfloat16")])
@pytest.mark.parametrize("T,Hin,Hout,n,R", SHAPES)
def test_against_the_plain_form(dtype, ydtype, T, Hin, Hout, n, R):
    Batch(T, Hin, Hout, n, R, dtype, ydtype, seed=T + R).check()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_ranks_of_their_own(dtype):
    """Adapters of ranks 0 to R in one batch."""
    Batch(200, 264, 136, 7, 64, dtype, ranks=[64, 1, 0, 16, 33, 8, 63], seed=3).check()
    Batch(20, 128, 128, 4, 128, dtype, ranks=[0, 0, 128, 5], seed=4).check()


@pytest.mark.parametrize("ids", ["one", "none", "outside", "runs", "last"])
def test_batches_of_one_kind(ids):
    import torch
    T, n = 150, 6
    kind = {"one": np.full(T, 3), "none": np.full(T, -1), "outside": np.where(np.arange(T) % 2, 2 ** 31 - 1, -2 ** 31),
            "runs": np.repeat(np.arange(6), 25), "last": np.full(T, n - 1)}[ids]
    b = Batch(T, 128, 192, n, 16, ids=kind, seed=5)
    b.check()
    if ids in ("none", "outside"):
        assert torch.equal(b.forward(), b.base)
        assert not b.forward(base=None).any()
        _, dA, dB = b.backward(torch.zeros((T, 16), device=DEV))
        assert not any(m.any() for m in dA + dB)


@pytest.mark.parametrize("T,n", [(1, 1), (63, 1), (1000, 4096), (1024, 7), (1025, 7), (5000, 1000), (65536, 3), (4097, 4096)])
def test_plan_sorts(T, n):
    """Through the operator: a rank-1 adapter whose factor tells adapters apart; every token gets its own."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    ids = torch.randint(-2, n + 2, (T,), generator=torch.Generator(device=DEV).manual_seed(T), device=DEV, dtype=torch.int32)
    plan = torch.empty(S.lora_plan_bytes(T, n), dtype=torch.uint8, device=DEV)
    S.lora_plan(ids, n, plan)
    A, B = torch.ones((1, 8), device=DEV), torch.arange(n, device=DEV).float()[:, None].repeat(1, 8) + 1
    ap = torch.full((n,), A.data_ptr(), dtype=torch.int64, device=DEV)
    bp = torch.tensor([B.data_ptr() + 32 * i for i in range(n)], dtype=torch.int64, device=DEV)
    x = (torch.arange(T, device=DEV) % 61).float()[:, None].repeat(1, 8)
    y = torch.full((T, 8), -7.0, device=DEV)
    ws = torch.empty(S.lora_workspace_bytes(T, 8, 8, n, 1, torch.float32), dtype=torch.uint8, device=DEV)
    S.lora(x, plan, ap, bp, 1, y, ws)
    ok = (ids >= 0) & (ids < n)
    assert torch.equal(y, torch.where(ok, 8 * x[:, 0] * (ids + 1), 0.0)[:, None].expand(T, 8))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("pad,off", [(0, 1), (8, 8), (5, 3), (64, 0)])
def test_strided_and_unaligned_rows(dtype, pad, off):
    Batch(70, 128, 256, 3, 16, dtype, seed=6, pad=pad, off=off).check()


def test_in_place_and_without_a_base():
    import torch
    for dtype, ydtype in (("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "float32")):
        b = Batch(90, 256, 136, 4, 16, dtype, ydtype, seed=8)
        want = b.forward()
        y = b.base.clone()
        assert torch.equal(b.forward(base=y, y=y), want)
        b.check_forward(b.forward(base=None), None, None)
        wide = torch.full((90, 200), 3.0, dtype=b.ydt, device=DEV)
        b.forward(y=wide[:, 32:168])
        assert torch.equal(wide[:, 32:168], want) and (wide[:, :32] == 3).all() and (wide[:, 168:] == 3).all()
        v = torch.empty((90, 16), device=DEV)
        b.forward(v=v)
        dx, dA, dB = b.backward(v)
        d = b.dbase.clone()
        got = b.backward(v, dx=d, base=d)
        assert torch.equal(got[0], dx) and all(torch.equal(p, q) for p, q in zip(got[1] + got[2], dA + dB))
        none = b.backward(v, dx=None)
        assert all(torch.equal(p, q) for p, q in zip(none[1] + none[2], dA + dB))
        b.check_backward(*b.backward(v, base=None), None)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,n", [(40, 3), (1100, 4)])
def test_infinite_and_nan_rows_stay_alone(dtype, T, n):
    """A token's infinities and NaN reach its own row (and its adapter's gradients) alone, also past the rank, the last
    column and the last token of a tile."""
    import torch
    ranks = [16, 5, 9, 3][:n]
    b = Batch(T, 264, 136, n, 16, dtype, ranks=ranks, seed=9)
    v = torch.empty((T, 16), device=DEV)
    y0 = b.forward(v=v)
    b.ids[7], b.ids[21] = 1, 1
    b.adapter.copy_(torch.from_numpy(b.ids))
    from paper_2606_15453_amd import stmoe as S
    S.lora_plan(b.adapter, n, b.plan)
    y0 = b.forward(v=v)
    _, dA0, dB0 = b.backward(v)
    b.x[7], b.dy[7] = float("inf"), float("inf")
    b.x[21, 3], b.dy[21, 0] = float("nan"), float("nan")
    v2 = torch.empty((T, 16), device=DEV)
    y = b.forward(v=v2)
    keep = [t for t in range(T) if t not in (7, 21)]
    assert torch.equal(y[keep], y0[keep]) and not torch.isfinite(y[7]).any() and torch.isnan(y[21]).all()
    assert not v2[7, 5:].any()
    dx0, dA, dB = b.backward(v2)
    assert torch.isfinite(dx0[keep]).all()
    for a in range(n):
        if a != 1:
            assert torch.equal(dA[a], dA0[a]) and torch.equal(dB[a], dB0[a])


def test_gradient_against_differences():
    """d sum(y . dy) along directions of x, A and B, by central differences of the plain form in 64 bits (h = 1e-4, and
    the third derivative of a product of two is zero)."""
    import torch
    b = Batch(120, 72, 56, 3, 9, "float32", seed=11)
    v = torch.empty((120, 9), device=DEV)
    b.forward(v=v)
    dx, dA, dB = b.backward(v, base=None)
    x, dy, s = _f64(b.x), _f64(b.dy), _f64(b.scales)
    A, B = [_f64(m) for m in b.A], [_f64(m) for m in b.B]
    f = lambda x_, A_, B_: (scoredref.lora(x_, b.ids, A_, B_, s, 0 * dy)[0] * dy).sum()
    r, h = np.random.RandomState(12), 1e-4
    for what in "xAB":
        px = r.randn(*x.shape) if what == "x" else 0 * x
        pA = [r.randn(*m.shape) if what == "A" else 0 * m for m in A]
        pB = [r.randn(*m.shape) if what == "B" else 0 * m for m in B]
        go = lambda e: f(x + e * px, [m + e * p for m, p in zip(A, pA)], [m + e * p for m, p in zip(B, pB)])
        want = (go(h) - go(-h)) / (2 * h)
        got = [(_f64(dx) * px)] + [_f64(m) * p for m, p in zip(dA, pA)] + [_f64(m) * p for m, p in zip(dB, pB)]
        size = sum(np.abs(m).sum() for m in got)
        assert abs(sum(m.sum() for m in got) - want) <= 1e-5 * size + 1e-7


def test_repeats_give_the_same_bits_and_larger_workspaces_do():
    import torch
    from paper_2606_15453_amd import stmoe as S
    b = Batch(3000, 512, 384, 5, 16, seed=13)
    v, v2 = torch.empty((3000, 16), device=DEV), torch.empty((3000, 16), device=DEV)
    y, g = b.forward(v=v), b.backward(v)
    b.ws.fill_(0x55)
    b.gws = torch.full((S.lora_backward_workspace_bytes(65536, 512, 384, 5, 16, b.dt),), 0x55, dtype=torch.uint8, device=DEV)
    own = (b.ids >= 0) & (b.ids < 5)
    assert torch.equal(b.forward(v=v2), y) and torch.equal(v[own], v2[own])
    g2 = b.backward(v)
    assert torch.equal(g2[0], g[0]) and all(torch.equal(p, q) for p, q in zip(g2[1] + g2[2], g[1] + g[2]))


def test_a_plan_of_another_batch_writes_nothing():
    import torch
    from paper_2606_15453_amd import stmoe as S
    b = Batch(40, 64, 64, 3, 8, seed=14)
    S.lora_plan(b.adapter[:30].contiguous(), 3, b.plan)
    y = torch.full((40, 64), 2.0, dtype=b.ydt, device=DEV)
    b.forward(y=y)
    assert (y == 2).all()
    _, dA, dB = b.backward(torch.zeros((40, 8), device=DEV))
    assert all(torch.isnan(m).all() for m in dA + dB)
    b.plan = b.plan[:1024].clone()
    with pytest.raises(S.StmoeError, match="plan too small"):
        b.forward(y=y)
    with pytest.raises(S.StmoeError, match="plan too small"):
        b.backward(torch.zeros((40, 8), device=DEV))


def test_the_gradient_of_x_does_not_take_its_place():
    from paper_2606_15453_amd import stmoe as S
    import torch
    b = Batch(8, 64, 64, 2, 8, seed=19)
    v = torch.zeros((8, 8), device=DEV)
    for bad in (b.x, b.dy):
        with pytest.raises(S.StmoeError):
            b.backward(v, dx=bad)


def test_streams_and_graphs():
    """On another stream; captured with the plan and replayed over new adapters and inputs between eager work."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    for T in (20, 1300):
        b = Batch(T, 256, 192, 4, 16, seed=15)
        v = torch.zeros((T, 16), device=DEV)
        want = b.forward(v=v)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        v1, y = torch.zeros_like(v), torch.empty_like(want)
        b.forward(y=y, v=v1, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(v1, v)
        dA, dB = [torch.empty((16, 256), device=DEV) for _ in range(4)], [torch.empty((16, 192), device=DEV) for _ in range(4)]
        ap, bp, dx = b.at(dA), b.at(dB), torch.empty((T, 256), dtype=b.dt, device=DEV)

        def step():
            S.lora_plan(b.adapter, 4, b.plan)
            b.forward(y=y, v=v1)
            S.lora_backward(b.x, b.dy, v1, b.plan, b.ap, b.bp, 16, ap, bp, b.gws, dx=dx, base=b.dbase, scales=b.scales)

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        r = np.random.RandomState(16)
        for _ in range(3):
            b.ids = r.randint(-1, 5, T).astype(np.int32)
            b.adapter.copy_(torch.from_numpy(b.ids))
            b.x.copy_(torch.randn((T, 256), device=DEV))
            y.fill_(0)
            g.replay()
            torch.cuda.synchronize()
            got = [m.clone() for m in [y, dx] + dA + dB]
            S.lora_plan(b.adapter, 4, b.plan)
            e = b.forward(v=v1)
            ex, eA, eB = b.backward(v1)
            assert all(torch.equal(p, q) for p, q in zip(got, [e, ex] + eA + eB))


def test_offsets_beyond_32_bits():
    """Rows 2^27 elements apart: offsets beyond 2^31 elements and 4 GiB in x, y, base, dy and dx."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    T, ld = 40, 1 << 27
    small = Batch(T, 64, 72, 2, 8, seed=17)
    v = torch.empty((T, 8), device=DEV)
    want, (dx, dA, dB) = small.forward(v=v), (None, None, None)
    dx, dA, dB = small.backward(v)
    far = lambda m: torch.empty((T - 1) * ld + m.shape[1], dtype=m.dtype, device=DEV).as_strided(m.shape, (ld, 1)).copy_(m)
    small.x, small.base = far(small.x), far(small.base)
    v2, y = torch.empty((T, 8), device=DEV), far(want)
    y.zero_()
    small.forward(y=y, v=v2)
    assert torch.equal(y, want)
    small.base = y = None
    small.dy, small.dbase = far(small.dy), far(small.dbase)
    gx, gA, gB = small.backward(v, dx=far(dx))
    assert torch.equal(gx, dx) and all(torch.equal(p, q) for p, q in zip(gA + gB, dA + dB))


def test_a_layer_with_adapters_end_to_end():
    """Router logits with an adapter, routed by scores, experts, an adapter beside the expert block; then the gradient of
    the weights through the router's adapter, and the bias's step: against the plain forms of each."""
    import torch
    import mxref
    from paper_2606_15453_amd import stmoe as S
    T, H, I, E, K, n, R = 24, 256, 128, 16, 4, 3, 8
    g = torch.Generator(device=DEV).manual_seed(20)
    rnd = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    wg = rnd(E, H) * H ** -0.5
    r = Batch(T, H, E, n, R, "bfloat16", "float32", seed=21)
    b = Batch(T, H, H, n, R, "bfloat16", "float32", ids=r.ids, seed=22)
    r.base = r.x.float() @ wg.T
    v = torch.zeros((T, R), device=DEV)
    logits = r.forward(v=v)
    r.check_forward(logits, v, r.base)
    bias, counts = torch.zeros(E, device=DEV), torch.zeros(E, dtype=torch.int32, device=DEV)
    idx, w = torch.empty((T, K), dtype=torch.int32, device=DEV), torch.empty((T, K), device=DEV)
    kw = dict(score="sigmoid", renorm=True, scale=2.0)
    S.route_scored(logits, K, idx, w, bias=bias, n_groups=4, top_groups=2, counts=counts, **kw)
    ri, rw, rc = scoredref.route(_f64(logits), K, "sigmoid", np.zeros(E), 4, 2, 2, True, 2.0)
    assert np.array_equal(idx.cpu().numpy(), ri) and np.array_equal(counts.cpu().numpy(), rc)
    # experts in 4 bits on that selection; the adapter beside them in place
    mats = [[rnd(I, H) * H ** -0.5, rnd(I, H) * H ** -0.5, rnd(H, I) * I ** -0.5] for _ in range(E)]
    blobs = torch.empty((E, S.blob_bytes(H, I, S.MXFP4)), dtype=torch.uint8, device=DEV)
    values = []
    for e in range(E):
        parts = []
        for m in mats[e]:
            codes = torch.empty((m.shape[0], m.shape[1] // 2), dtype=torch.uint8, device=DEV)
            scales = torch.empty((m.shape[0], m.shape[1] // 32), dtype=torch.uint8, device=DEV)
            S.mx_quantize(m, codes, scales)
            parts.append((codes, scales))
        S.mx_pack_expert(*parts, H, I, blobs[e])
        values.append([mxref.mx_values(c.cpu().numpy(), s.cpu().numpy(), 2 * c.shape[1]) for c, s in parts])
    ptrs = torch.tensor([blobs[e].data_ptr() for e in range(E)], dtype=torch.int64, device=DEV)
    y = torch.empty((T, H), device=DEV)
    b.x = r.x
    ws = torch.empty(S.ffn_mx_workspace_bytes(T, K, E, H, I), dtype=torch.uint8, device=DEV)
    S.expert_ffn_mx(b.x, idx, w, H, I, E, ptrs, y, ws)
    ffn = mxref.moe_ffn(_f64(b.x), ri, rw, values)
    assert np.linalg.norm(_f64(y) - ffn) <= 1e-5 * np.linalg.norm(ffn)
    b.base = y.clone()
    b.forward(base=y, y=y)
    b.check_forward(y, None, b.base)
    # back: the weights' gradient to the logits, through the router's adapter
    d_w, d_z = rnd(T, K), torch.empty((T, E), device=DEV)
    S.route_scored_backward(logits, idx, d_w, d_z, **kw)
    rz = scoredref.route_grad(_f64(logits), ri, _f64(d_w), "sigmoid", True, 2.0)
    assert np.abs(_f64(d_z) - rz).max() <= 1e-5 * np.abs(_f64(d_w)).max()
    r.dy = d_z.bfloat16()
    r.check_backward(*r.backward(v), r.dbase)
    S.route_bias_step(counts, bias, 1e-3, reset=True)
    np.testing.assert_allclose(_f64(bias), scoredref.bias_step(rc, np.zeros(E), 1e-3), rtol=2.0 ** -23)
