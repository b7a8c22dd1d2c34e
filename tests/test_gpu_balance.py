"""GPU: the router of a batch (top-K, counts, balance and z loss) and its
gradient against the plain 64-bit forms.

Tolerances.  A row's exponentials take z - max, rounded to 2^-24 of at most
about 40: 2.4e-6 relative, and expf's own 2^-23; probabilities and weights are
quotients of such terms: 5e-6 relative.  lse^2: 2^-23 of the logarithm twice.
A gradient is p times a difference of terms, each with that error: 1e-5 of the
largest term of its row; a bf16 result adds 2^-8 of itself."""
import numpy as np
import pytest

import mxref

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


def _forward(z, K, renorm=False, mask=None, stream=None, ws=None):
    import torch
    from paper_2606_15453_amd import stmoe as S
    T, E = z.shape
    o = dict(idx=torch.full((T, K), 77, dtype=torch.int32, device=DEV), w=torch.full((T, K), float("nan"), device=DEV),
             counts=torch.full((E,), -5, dtype=torch.int32, device=DEV), n=torch.full((1,), -5, dtype=torch.int32, device=DEV),
             loss=torch.full((2,), float("nan"), device=DEV), prob_sum=torch.full((E,), float("nan"), device=DEV))
    if ws is None:
        ws = torch.full((S.route_balance_workspace_bytes(T, E),), 0xFF, dtype=torch.uint8, device=DEV)
    S.route_balance(z, K, o["idx"], o["w"], o["counts"], o["n"], o["loss"], ws, renorm=renorm, mask=mask,
                    prob_sum=o["prob_sum"], stream=stream)
    return o


def _check_forward(z, K, renorm=False, mask=None):
    o = _forward(z, K, renorm, mask)
    f = mxref.balance(_f64(z), K, renorm, None if mask is None else mask.cpu().numpy())
    assert np.array_equal(o["idx"].cpu().numpy(), f["idx"])
    assert np.array_equal(o["counts"].cpu().numpy(), f["counts"])
    assert int(o["n"]) == f["n"]
    np.testing.assert_allclose(_f64(o["w"]), f["w"], rtol=5e-6, atol=1e-30)
    np.testing.assert_allclose(_f64(o["prob_sum"]), f["prob_sum"], rtol=6e-6, atol=1e-30)
    # in fp32: a row at fp32's lowest value has lse^2 = 1.2e77, which rounds to infinity (the largest fp32 is 3.4e38)
    with np.errstate(over="ignore"):
        want = f["loss"].astype(np.float32)
    np.testing.assert_allclose(_f64(o["loss"]), want, rtol=1e-5, atol=1e-12)
    return o, f


def _backward(z, f, d_w, d_loss, renorm, out=None, stream=None):
    import torch
    from paper_2606_15453_amd import stmoe as S
    i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32).copy()).to(DEV)      # noqa: E731
    d = torch.full(z.shape, float("nan"), dtype=z.dtype, device=DEV) if out is None else out
    S.route_balance_backward(z, i32(f["idx"]), i32(f["counts"]), i32([f["n"]]),
                             torch.tensor(d_loss, dtype=torch.float32, device=DEV), d,
                             d_w=None if d_w is None else torch.from_numpy(d_w.astype(np.float32)).to(DEV), renorm=renorm,
                             stream=stream)
    return d


def _check_backward(z, f, d_w, d_loss, renorm):
    zz = _f64(z)
    want = mxref.balance_grad(zz, f["idx"], f["counts"], f["n"], d_w if d_w is not None else np.zeros(f["idx"].shape),
                              np.float32(d_loss).astype(np.float64), renorm)
    got = _f64(_backward(z, f, d_w, d_loss, renorm))
    # the terms of a row before they cancel: p times the largest coefficient, the z loss's, and with renormalised
    # weights those of the selected experts
    n = max(f["n"], 1)
    c = d_loss[0] * zz.shape[1] * f["counts"].max(initial=0) / (n * n * f["idx"].shape[1])
    big = c + 2 * abs(d_loss[1]) / n * np.abs(f["lse"]) + (np.abs(d_w).max(axis=1) if d_w is not None else 0)
    tol = 1e-5 * big[:, None] * (f["prob"] + (1 if renorm else 0)) + 1e-30
    import torch
    if z.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(want)
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
    return got


SHAPES = [(1, 1, 1), (1, 8, 2), (3, 2, 2), (5, 31, 4), (7, 32, 3), (4, 33, 5), (64, 64, 8), (130, 61, 4), (33, 100, 7),
          (257, 128, 8), (50, 129, 16), (20, 256, 16), (11, 200, 1), (2100, 16, 2)]


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,E,K", SHAPES)
def test_balance_and_gradient(T, E, K, dtype, renorm):
    import torch
    rng = np.random.default_rng(T * E + K)
    z = _logits(T, E, T + E, dtype)
    mask = torch.from_numpy((rng.random(T) < 0.8).astype(np.uint8)).to(DEV) if T % 2 else None
    _, f = _check_forward(z, K, renorm, mask)
    d_w = rng.normal(size=(T, K)).astype(np.float32).astype(np.float64)
    _check_backward(z, f, d_w, [0.5, 0.25], renorm)
    _check_backward(z, f, None, [1.0, 0.0], renorm)
    _check_backward(z, f, d_w, [0.0, 0.0], renorm)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_ties_go_to_the_lower_index(dtype):
    import torch
    z = torch.zeros((40, 96), device=DEV)
    z[10:20, 1::2] = 1.0
    z[20:30] = torch.arange(96, device=DEV) // 7 % 3
    z[30:, 5], z[30:, 70] = -0.0, 0.0
    for E in (96, 64, 40, 32, 12):
        _check_forward(z.to(getattr(torch, dtype))[:, :E].contiguous(), 6)


@pytest.mark.parametrize("E", [20, 64, 150])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_masked_experts_and_tokens(dtype, E):
    """Minus infinity in some, in all but fewer than K, in all places; the type's lowest value; tokens masked out whose
    logits are NaN; bool masks."""
    import torch
    dt = getattr(torch, dtype)
    K, T = 5, 48
    z = _logits(T, E, E, dtype).clone()
    low = torch.finfo(dt).min
    z[0, ::2] = -float("inf")
    z[1, 3:] = -float("inf")                 # fewer candidates than K
    z[2] = -float("inf")                     # none
    z[3, 1:] = low
    z[4] = low                               # a row of equal numbers
    z[5, 4:] = low
    z[6] = float("nan")
    z[7] = -float("inf")
    z[8, E - 1] = -float("inf")
    mask = torch.ones(T, dtype=torch.bool, device=DEV)
    mask[6] = mask[7] = mask[11] = False
    o, f = _check_forward(z, K, True, mask)
    assert o["idx"][2].tolist() == [-1] * K and o["idx"][1, 3:].tolist() == [-1, -1] and o["idx"][4].tolist() == list(range(K))
    d_w = np.random.default_rng(0).normal(size=(T, K))
    z0, keep = _f64(z), f["live"]
    rows = np.nonzero(keep)[0]
    got = _f64(_backward(z, f, d_w, [0.5, 0.0], True))
    assert not got[~keep].any() and np.isfinite(got).all()
    assert not got[z0 == -np.inf].any()
    want = mxref.balance_grad(np.where(keep[:, None], z0, 0), f["idx"], f["counts"], f["n"],
                              d_w.astype(np.float32).astype(np.float64), [0.5, 0.0], True)
    tol = 1e-5 * (1 + np.abs(d_w).max()) + (2.0 ** -8 * np.abs(want) if dtype == "bfloat16" else 0)
    assert (np.abs(got - want) <= tol)[rows].all()


def test_no_live_token():
    import torch
    z = _logits(9, 24, 1, "float32")
    mask = torch.zeros(9, dtype=torch.uint8, device=DEV)
    o, f = _check_forward(z, 3, False, mask)
    assert int(o["n"]) == 0 and not o["loss"].any() and bool((o["idx"] == -1).all())
    assert not _backward(z, f, None, [1.0, 1.0], False).any()
    o = _forward(z[:0], 3)
    assert int(o["n"]) == 0 and not o["counts"].any() and not o["loss"].any() and not o["prob_sum"].any()


def test_nan_and_infinity_show():
    """A NaN or +infinity in a live row: that row's weights and the losses are NaN, the other rows are untouched; a NaN
    is selected only after the numbers."""
    import torch
    z = _logits(6, 40, 2, "float32").clone()
    clean = _forward(z, 4)
    z[1, 7], z[3, 2], z[4, 1:] = float("nan"), float("inf"), float("nan")
    o = _forward(z, 4)
    for r in (0, 2, 5):
        assert torch.equal(o["idx"][r], clean["idx"][r]) and torch.equal(o["w"][r], clean["w"][r])
    assert 7 not in o["idx"][1].tolist() and int(o["idx"][3, 0]) == 2 and o["idx"][4].tolist() == [0, 1, 2, 3]
    assert bool(o["loss"].isnan().all()) and bool(o["w"][1].isnan().all()) and int(o["n"]) == 6


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("ld,off", [(61, 0), (64, 0), (64, 1), (70, 3)])
def test_strided_logits(dtype, ld, off):
    import torch
    z = _logits(77, 61, 5, dtype, ld, off)
    _, f = _check_forward(z, 4, True)
    d_w = np.random.default_rng(1).normal(size=(77, 4)).astype(np.float32).astype(np.float64)
    want = _backward(z.contiguous(), f, d_w, [0.5, 0.1], True)
    base = torch.full((77 * ld + off,), 7.0, dtype=z.dtype, device=DEV)
    d = base[off:].view(77, ld)
    _backward(z, f, d_w, [0.5, 0.1], True, out=d[:, :61])
    assert torch.equal(d[:, :61], want)
    assert bool((d[:, 61:] == 7).all()) and bool((base[:off] == 7).all())


def test_gradient_in_place():
    import torch
    z = _logits(50, 40, 6, "float32").clone()
    _, f = _check_forward(z, 4)
    want = _backward(z, f, None, [1.0, 0.5], False)
    _backward(z, f, None, [1.0, 0.5], False, out=z)
    assert torch.equal(z, want)


def test_many_tokens_same_bits_and_streams():
    """A batch beyond one round of workgroups, on a stream of its own, twice: the same bits; sums against 64 bits."""
    import torch
    z = _logits(20000, 64, 7, "float32")
    a = _forward(z, 6, True)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = _forward(z, 6, True, stream=s)
    s.synchronize()
    assert all(torch.equal(a[k], b[k]) for k in a)
    p = torch.softmax(z.double(), dim=1)
    np.testing.assert_allclose(_f64(a["prob_sum"]), p.sum(dim=0).cpu().numpy(), rtol=6e-6)
    assert int(a["counts"].sum()) == 6 * 20000


def test_captured_and_replayed():
    """Forward and backward in one graph, replayed on changing logits with eager work between, equal the eager calls."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    T, E, K = 300, 48, 4
    z = _logits(T, E, 1, "float32").clone()
    o = _forward(z, K)
    ws = torch.empty(S.route_balance_workspace_bytes(T, E), dtype=torch.uint8, device=DEV)
    d, d_loss = torch.empty_like(z), torch.tensor([1.0, 0.5], device=DEV)
    d_w = torch.randn((T, K), device=DEV)

    def step(z, o, ws, d):
        S.route_balance(z, K, o["idx"], o["w"], o["counts"], o["n"], o["loss"], ws, prob_sum=o["prob_sum"])
        S.route_balance_backward(z, o["idx"], o["counts"], o["n"], d_loss, d, d_w=d_w)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(z, o, ws, d)
    for seed in range(4):
        z.copy_(_logits(T, E, 50 + seed, "float32"))
        e = {k: torch.empty_like(v) for k, v in o.items()}
        de = torch.empty_like(z)
        step(z, e, torch.empty_like(ws), de)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(d, de) and all(torch.equal(o[k], e[k]) for k in o), seed


def test_layer_of_a_training_batch():
    """The operators as they are used together: router logits, selection with padding tokens, 4-bit experts on the
    selection, and the router's gradient from the gate weights' own gradient."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    from test_gpu_mx import Experts, _err, _run
    T, H, I, E, K = 150, 256, 136, 12, 3
    ex = Experts(E, H, I, 1)
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.randn((T, H), generator=g, device=DEV).to(torch.bfloat16)
    z = (x.float() @ torch.randn((H, E), generator=g, device=DEV) * H ** -0.5)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[140:] = 0
    o, f = _check_forward(z, K, True, mask)
    y = _run(ex, E, H, I, x, o["idx"], o["w"], torch.float32)
    want = mxref.moe_ffn(_f64(x), f["idx"], _f64(o["w"]), ex.values)
    assert _err(y, want) <= 2e-5 and not y[140:].any()
    # loss = sum(y * r): the gradient of gate weight k is r . (expert output k), here from 64 bits
    r = np.random.default_rng(0).normal(size=(T, H))
    d_w = np.zeros((T, K))
    for k in range(K):
        one = np.full((T, K), -1)
        one[:, k] = f["idx"][:, k]
        d_w[:, k] = (mxref.moe_ffn(_f64(x), one, np.ones((T, K)), ex.values) * r).sum(axis=1)
    d_w = d_w.astype(np.float32).astype(np.float64)
    got = _check_backward(z, f, d_w, [0.01, 0.001], True)
    assert not got[140:].any()


@pytest.mark.parametrize("T,E,dtype", [(2 ** 26, 3, "bfloat16"), (2 ** 24, 61, "bfloat16"), (2 ** 24, 61, "float32"),
                                       (2 ** 24, 124, "bfloat16"), (2 ** 24, 200, "bfloat16")])
def test_sums_of_the_largest_batches(T, E, dtype):
    """Rows of equal logits, as a fresh router gives them, whose rounding errors do not cancel.  In half steps of 2^-24:
    a row's probability is off by two, a chain of 32 rows, four rows side by side and 16 waves by 49 more, a product
    and the last rounding by two; the logarithm's square by eight."""
    import torch
    K = 2
    z = torch.zeros((T, E), dtype=getattr(torch, dtype), device=DEV)
    o = _forward(z, K)
    u = 2.0 ** -24
    np.testing.assert_allclose(_f64(o["prob_sum"]), np.full(E, T / E), rtol=53 * u)
    loss = _f64(o["loss"])
    assert abs(loss[0] - 1) <= 53 * u and abs(loss[1] / np.log(E) ** 2 - 1) <= 59 * u
    assert o["counts"].tolist() == [T, T] + [0] * (E - 2) and int(o["n"]) == T


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T", [12, 150])
def test_router_gradient_from_the_experts_own_outputs(T, renorm):
    """A gate weight's gradient is dy . (its expert's own output), and expert_ffn_mx over one column of the selection
    with weights of one gives those outputs: the router's gradient from the library's own calls alone, against 64 bits.
    A column's outputs are off by 2e-5 of their norm and the fp32 product of H terms by H 2^-24 of theirs; a row of the
    gradient takes at most twice the largest of its K errors."""
    import torch
    from test_gpu_mx import Experts, _run
    H, I, E, K = 256, 136, 12, 3
    ex = Experts(E, H, I, 1)
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randn((T, H), generator=g, device=DEV).to(torch.bfloat16)
    z = x.float() @ torch.randn((H, E), generator=g, device=DEV) * H ** -0.5
    r = torch.randn((T, H), generator=g, device=DEV)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[-2:] = 0
    o, f = _check_forward(z, K, renorm, mask)
    ones = torch.ones((T, 1), device=DEV)
    d_w = torch.stack([(_run(ex, E, H, I, x, o["idx"][:, k:k + 1].contiguous(), ones, torch.float32) * r).sum(dim=1)
                       for k in range(K)], dim=1)
    want_w, off = np.zeros((T, K)), np.zeros((T, K))
    for k in range(K):
        out = mxref.moe_ffn(_f64(x), f["idx"][:, k:k + 1], np.ones((T, 1)), ex.values)
        want_w[:, k] = (out * _f64(r)).sum(axis=1)
        off[:, k] = (2e-5 + H * 2.0 ** -24) * np.linalg.norm(out, axis=1) * np.linalg.norm(_f64(r), axis=1)
    assert (np.abs(_f64(d_w) - want_w) <= off).all()
    d_loss = [0.01, 0.001]
    got = _f64(_backward(z, f, _f64(d_w), d_loss, renorm))
    want = mxref.balance_grad(_f64(z), f["idx"], f["counts"], f["n"], want_w, np.float32(d_loss).astype(np.float64), renorm)
    big = np.abs(want_w).max(axis=1) + d_loss[0] * E + 2 * d_loss[1] * np.abs(f["lse"])
    assert (np.abs(got - want) <= (2 * off.max(axis=1) + 1e-5 * 2 * big)[:, None]).all()
    assert not got[-2:].any() and np.abs(got).max() > 1e-3
