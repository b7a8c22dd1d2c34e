"""4-bit experts and the balanced router without a GPU: refusals before any
device work, size queries, and the plain forms the GPU tests compare with."""
import numpy as np
import pytest

import mxref

S = pytest.importorskip("paper_2606_15453_amd.stmoe")
L = S._lib


def test_blob_bytes():
    # 16-row x 128-column tiles of 1024 bytes; scales in groups of four tiles, 256 bytes
    assert S.blob_bytes(2048, 768, S.MXFP4) == 3 * (48 * 16 * 1024) + 2 * 48 * 4 * 256 + 128 * 2 * 256
    assert S.blob_bytes(8, 8, S.MXFP4) == 3 * (1024 + 256)
    assert S.blob_bytes(4096, 14336, S.MXFP4) * 3.7 < S.blob_bytes(4096, 14336, S.BF16)
    for H, I in [(12, 64), (64, 12), (16392, 64), (64, 65544), (0, 64)]:
        assert S.blob_bytes(H, I, S.MXFP4) == 0
    assert S.blob_bytes(64, 64, 3) == 0


def test_quantize_refusals():
    q, d = L.moe_mx_quantize, L.moe_mx_dequantize
    ok = dict(x=256, rows=4, cols=64, ld=64, dt=S.BF16, codes=256, scales=256)
    for bad in [dict(x=None), dict(codes=None), dict(scales=None), dict(rows=-1), dict(rows=2 ** 31 + 1), dict(cols=0),
                dict(cols=2 ** 30 + 1), dict(ld=63), dict(dt=S.MXFP4), dict(dt=7), dict(x=257), dict(x=258, dt=S.F32)]:
        a = dict(ok, **bad)
        assert q(a["x"], a["rows"], a["cols"], a["ld"], a["dt"], a["codes"], a["scales"], None) == S.EINVAL, bad
        assert d(a["codes"], a["scales"], a["rows"], a["cols"], a["x"], a["ld"], a["dt"], None) == S.EINVAL, bad
        assert L.stmoe_last_error().decode().startswith("moe_mx_dequantize:")
    assert q(None, 0, 64, 64, S.BF16, None, None, None) == S.OK      # no rows: nothing to do
    assert d(None, None, 0, 64, None, 64, S.F32, None) == S.OK


def test_pack_refusals():
    p = L.moe_mx_pack_expert
    for i in range(7):
        a = [256] * 6 + [64, 64] + [256]
        a[i if i < 6 else 8] = None
        assert p(*a, None) == S.EINVAL
    for H, I, out in [(60, 64, 256), (64, 60, 256), (16392, 64, 256), (64, 65544, 256), (64, 64, 264)]:
        assert p(256, 256, 256, 256, 256, 256, H, I, out, None) == S.EINVAL
    # the host packer takes row-major storage only
    assert L.moe_pack_expert(256, 256, 256, 64, 64, S.MXFP4, 256) == S.EINVAL


def test_ffn_refusals():
    f = L.moe_expert_ffn_mx
    ok = dict(x=256, idx=256, w=256, T=4, K=2, H=64, I=64, E=8, dt=S.BF16, yt=S.F32, ep=256, sp=None, ns=0, y=256,
              ws=256, n=1 << 30)
    for bad in [dict(x=None), dict(idx=None), dict(w=None), dict(ep=None), dict(y=None), dict(ws=None), dict(T=-1),
                dict(T=65537), dict(K=0), dict(K=9), dict(K=17, E=32), dict(H=12), dict(H=16392), dict(H=0), dict(I=4),
                dict(I=65544), dict(E=0), dict(E=257), dict(dt=S.MXFP4), dict(yt=2), dict(ns=-1), dict(ns=9, sp=256),
                dict(ns=1), dict(n=1024), dict(x=264), dict(y=260), dict(ws=264)]:
        a = dict(ok, **bad)
        rc = f(a["x"], a["idx"], a["w"], a["T"], a["K"], a["H"], a["I"], a["E"], a["dt"], a["yt"], a["ep"], a["sp"],
               a["ns"], a["y"], a["ws"], a["n"], None)
        assert rc == S.EINVAL, bad
    assert f(None, None, None, 0, 2, 64, 64, 8, S.BF16, S.F32, None, None, 0, None, None, 0, None) == S.OK
    n = L.moe_expert_ffn_mx_workspace_bytes
    assert n(4, 2, 8, 64, 64, 0, S.BF16, S.F32) > 0
    for a in [(-1, 2, 8, 64, 64, 0, 1, 0), (65537, 2, 8, 64, 64, 0, 1, 0), (4, 9, 8, 64, 64, 0, 1, 0),
              (4, 2, 8, 60, 64, 0, 1, 0), (4, 2, 8, 64, 64, 9, 1, 0), (4, 2, 8, 64, 64, 0, 2, 0), (4, 2, 8, 64, 64, 0, 1, 2)]:
        assert n(*a) == 0
    # activations beyond 64 GiB (the launches count their 16-byte chunks in 32 bits)
    assert n(65536, 16, 16, 64, 32768, 0, S.BF16, S.BF16) > 0
    big = (65536, 16, 16, 64, 32776, 0, S.BF16, S.BF16)
    assert n(*big) == 0 and n(*big[:4], 10928, 0, S.BF16, S.F32) == 0 and n(*big[:4], 10920, 0, S.BF16, S.F32) > 0
    assert f(256, 256, 256, 65536, 16, 64, 32776, 16, S.BF16, S.BF16, 256, None, 0, 256, 256, 1 << 62, None) == S.EINVAL
    # pointers that their elements do not allow
    for bad in [dict(idx=258), dict(w=258), dict(ep=260), dict(ns=1, sp=260)]:
        a = dict(ok, **bad)
        assert f(a["x"], a["idx"], a["w"], a["T"], a["K"], a["H"], a["I"], a["E"], a["dt"], a["yt"], a["ep"], a["sp"],
                 a["ns"], a["y"], a["ws"], a["n"], None) == S.EINVAL, bad
    # the other FFN entries keep to row-major blobs
    assert L.moe_expert_ffn(256, 256, 256, 1, 2, 64, 64, 8, S.MXFP4, 256, None, 0, 256, 256, 1 << 30, None) == S.EINVAL


def test_balance_refusals():
    f, g = L.moe_route_balance, L.moe_route_balance_backward
    ok = dict(z=256, T=4, ld=8, E=8, K=2, dt=S.F32, idx=256, w=256, c=256, n=256, loss=256, ws=256, b=1 << 20)
    for bad in [dict(z=None), dict(T=-1), dict(T=2 ** 26 + 1), dict(ld=7), dict(E=0), dict(E=257, ld=257), dict(K=0),
                dict(K=9), dict(K=17, E=32, ld=32), dict(dt=2), dict(idx=None), dict(w=None), dict(c=None), dict(n=None),
                dict(loss=None), dict(ws=None), dict(ws=264), dict(b=16), dict(z=258)]:
        a = dict(ok, **bad)
        assert f(a["z"], a["T"], a["ld"], a["E"], a["K"], a["dt"], 0, None, a["idx"], a["w"], a["c"], a["n"], None,
                 a["loss"], a["ws"], a["b"], None) == S.EINVAL, bad
    ok = dict(z=256, T=4, ld=8, E=8, K=2, dt=S.F32, idx=256, c=256, n=256, dl=256, d=256, ldd=8)
    for bad in [dict(z=None), dict(T=-1), dict(ld=7), dict(ldd=7), dict(E=257, ld=257, ldd=257), dict(K=0), dict(dt=2),
                dict(idx=None), dict(c=None), dict(n=None), dict(dl=None), dict(d=None), dict(d=258)]:
        a = dict(ok, **bad)
        assert g(a["z"], a["T"], a["ld"], a["E"], a["K"], a["dt"], 0, a["idx"], a["c"], a["n"], None, a["dl"], a["d"],
                 a["ldd"], None) == S.EINVAL, bad
    assert g(None, 0, 8, 8, 2, S.F32, 0, None, None, None, None, None, None, 8, None) == S.OK
    assert L.moe_route_balance_workspace_bytes(0, 8) > 0
    assert L.moe_route_balance_workspace_bytes(4, 257) == 0


def test_binding_refuses_tensors_it_would_misread():
    import torch
    x = torch.zeros((4, 64))
    with pytest.raises(ValueError):      # not on the GPU
        S.mx_quantize(x, torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8))
    with pytest.raises(ValueError):
        S.route_balance(x, 2, *[x] * 6)
    with pytest.raises(ValueError):
        S.expert_ffn_mx(x, torch.zeros((4, 2), dtype=torch.int32), x, 64, 64, 8, x, x, x)


def test_plain_quantize_by_hand():
    # largest magnitude 10: scale 2^(3 - 2) = 2; 7 / 2 = 3.5 is a tie of 3 and 4, to the even code (4)
    x = np.zeros((1, 33))
    x[0, :8] = [10, -7, 5, 3, 1, 0.5, -0.49, 15.9]
    x[0, 32] = 2.0 ** -140
    c, s, v = mxref.mx_quantize(x)
    assert s.tolist() == [[128, 0]]
    assert v[0, :8].tolist() == [8, -8, 4, 3, 1, 0, -0.0, 12]      # 15.9 saturates at 6 * 2; 5 / 2 ties 2 and 3: 2
    assert v[0, 32] == 0
    assert c[0, :4].tolist() == [6 | 14 << 4, 4 | 3 << 4, 1 | 0 << 4, 8 | 7 << 4]
    assert np.array_equal(mxref.mx_values(c, s, 33)[0, :8], v[0, :8])


@pytest.mark.parametrize("renorm", [False, True])
def test_plain_gradient_against_differences(renorm):
    rng = np.random.default_rng(3 + renorm)
    T, E, K = 5, 7, 3
    z = rng.normal(0, 1.5, (T, E))
    f = mxref.balance(z, K, renorm, mask=[1, 1, 0, 1, 1])
    d_w, d_loss = rng.normal(size=(T, K)), np.array([0.7, 0.3])
    g = mxref.balance_grad(z, f["idx"], f["counts"], f["n"], d_w, d_loss, renorm)
    assert not g[2].any()
    num = np.zeros_like(z)
    h = 1e-5
    for t in range(T):
        for e in range(E):
            zp, zm = z.copy(), z.copy()
            zp[t, e] += h
            zm[t, e] -= h
            num[t, e] = (mxref.balance_total(zp, f["idx"], f["counts"], f["n"], d_w, d_loss, renorm)
                         - mxref.balance_total(zm, f["idx"], f["counts"], f["n"], d_w, d_loss, renorm)) / (2 * h)
    # central differences: h^2 / 6 times third derivatives of order 1-10, and 2^-52 / h
    assert np.abs(g - num).max() < 1e-8


def test_plain_losses_by_hand():
    # two experts, both tokens choose expert 0 with probability 3/4: balance = 2 * (1 * 3/4 + 0) = 1.5
    z = np.log(np.array([[3.0, 1.0], [3.0, 1.0]]))
    f = mxref.balance(z, 1)
    assert f["counts"].tolist() == [2, 0] and f["n"] == 2
    assert np.allclose(f["loss"], [1.5, np.log(4) ** 2], rtol=1e-14)


class _OnCard:
    """A tensor as the binding sees it: what its checks ask for, and an address."""

    def __init__(self, shape, dtype, device=0, step=1):
        import torch
        self.shape, self.dtype, self.device, self.step = torch.Size(shape), dtype, device, step
        self.nbytes = torch.empty(0, dtype=dtype).element_size() * self.shape.numel()

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.step == 1

    def dim(self):
        return len(self.shape)

    def stride(self):
        return tuple(self.shape[i + 1:].numel() * self.step for i in range(len(self.shape)))

    def data_ptr(self):
        return 4096

    def numel(self):
        return self.shape.numel()


@pytest.mark.parametrize("ws", [dict(device=-1), dict(device=1), dict(step=2), None])
def test_binding_refuses_workspaces_it_would_misread(monkeypatch, ws):
    """A workspace in host memory, on another GPU, with gaps between its elements, or none: no call goes to the library."""
    import torch
    calls = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(S, "_call", lambda name, *a: calls.append(name))
    monkeypatch.setattr(S, "_s", lambda stream: None)
    f, i, b = torch.float32, torch.int32, torch.bfloat16
    T, E, K, H, I = 4, 8, 2, 64, 64

    def run(w):
        S.route_balance(_OnCard((T, E), f), K, _OnCard((T, K), i), _OnCard((T, K), f), _OnCard((E,), i), _OnCard((1,), i),
                        _OnCard((2,), f), w)

    def ffn(w):
        S.expert_ffn_mx(_OnCard((T, H), b), _OnCard((T, K), i), _OnCard((T, K), f), H, I, E, _OnCard((E,), torch.int64),
                        _OnCard((T, H), f), w)

    good = _OnCard((1 << 20,), torch.uint8)
    run(good), ffn(good)
    assert calls == ["moe_route_balance", "moe_expert_ffn_mx"]
    bad = None if ws is None else _OnCard((1 << 20,), torch.uint8, **ws)
    for call in (run, ffn):
        with pytest.raises(ValueError):
            call(bad)
    assert len(calls) == 2


@pytest.mark.parametrize("xd", [S.BF16, S.F32])
@pytest.mark.parametrize("yd", [S.BF16, S.F32])
@pytest.mark.parametrize("K,E,H,I,ns", [(2, 8, 4096, 14336, 0), (8, 128, 2048, 768, 0), (6, 64, 2048, 1408, 2), (3, 13, 1000, 520, 1),
                                        (1, 1, 8, 8, 0), (16, 16, 16384, 64, 8), (1, 256, 256, 65536, 0), (2, 4, 64, 8192, 0)])
def test_a_workspace_for_many_tokens_serves_fewer(K, E, H, I, ns, xd, yd):
    n = L.moe_expert_ffn_mx_workspace_bytes
    rng = np.random.default_rng(K * E)
    sizes = sorted(set(range(0, 1100)) | set(rng.integers(1100, 65537, 3000).tolist()) | {65536})
    last = 0
    for T in sizes:
        b = n(T, K, E, H, I, ns, xd, yd)
        if b == 0:      # beyond the bound on the activations, which only larger batches are
            assert T * (K + ns) * I > 2 ** 35 // 3
            break
        assert b >= last, T
        last = b
    # not by far more than what the call writes: activations, terms in up to 64 parts of the contraction, x in pieces
    assert n(64, 2, 8, 4096, 14336, 0, xd, yd) <= 64 << 20
