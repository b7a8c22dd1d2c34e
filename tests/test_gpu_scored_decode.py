"""GPU: decode contexts that route by scores (moe_ctx_set_routing), resident and capped, eager and replayed: the
selections are moe_route_scored's on the router's logits, the predictor and the cache see them, and every layer's output
is the expert FFN's on them (against 64 bits, within the FFN tests' 1e-2)."""
import numpy as np
import pytest

import scoredref
from test_gpu_decode import Stack

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _context(st, capped, device, graph, renorm):
    import torch
    from gpuhelp import storage_dtype
    from paper_2606_15453_amd import stmoe as S
    cfg = st.cfg
    pred = S.Predictor(cfg.L, cfg.E, cfg.K, cfg.B)
    pred.profile(st.prof)
    keep = [pred]
    kw = dict(predictor=pred, shared_ptrs=st.shared_ptrs(), n_shared=cfg.n_shared, renorm=renorm)
    if capped:
        host = [st.blobs[l][e].cpu().pin_memory() for l in range(cfg.L) for e in range(cfg.E)]
        n_stage = max(1, min(cfg.B * cfg.K, cfg.E) - cfg.C)
        arena = torch.empty(S.cache_arena_bytes(cfg.L, cfg.E, cfg.C, cfg.blob_bytes, n_stage), dtype=torch.uint8, device=DEV)
        cache = S.ExpertCache(cfg.L, cfg.E, cfg.C, cfg.blob_bytes, n_stage, arena, [h.data_ptr() for h in host],
                              torch.cuda.Stream(), torch.cuda.Stream())
        cache.warm(st.warm)
        cache.set_device_policy(device)
        keep += [host, arena, cache]
        kw["cache"] = cache
    else:
        kw["resident_ptrs"] = [st.blobs[l][e].data_ptr() for l in range(cfg.L) for e in range(cfg.E)]
    ctx = S.DecodeContext(cfg.L, cfg.E, cfg.K, cfg.B, cfg.H, cfg.I, storage_dtype(cfg), [g.data_ptr() for g in st.wg_dev], **kw)
    if graph:
        ctx.set_graph(True)
    return ctx, pred, keep


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("over,score,groups,top,renorm", [
    (dict(B=1, T=6), "sigmoid", 4, 2, True), (dict(B=3, T=5, E=16, K=4, C=6), "sigmoid", 4, 2, False),
    (dict(B=2, T=5, n_shared=1), "softmax", 1, 1, True)])
def test_tokens(mode, over, score, groups, top, renorm):
    import torch
    from gpuhelp import expert_f64
    from oracle.stmoe_oracle import decode_storage, moe_ffn
    from paper_2606_15453_amd import stmoe as S
    from paper_2606_15453_amd import workload as W
    st = Stack(W.CONFIGS["tiny"].scaled(P=8, **over))
    cfg = st.cfg
    bias = torch.randint(-300, 301, (cfg.L, cfg.E), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) * 1e-3
    bias[1, 0] = -float("inf")
    outs = []
    for capped, device, graph in [(0, 0, 0), (0, 0, 1), (1, 0, 0), (1, 1, 0), (1, 1, 1)]:
        ctx, pred, keep = _context(st, capped, device, graph, renorm)
        ctx.set_routing(score, bias, groups, top, 2, 1.5)
        run = []
        for t in range(cfg.T):
            y = torch.full((cfg.L, cfg.B, cfg.H), float("nan"), device=DEV)
            ctx.token(t, st.x_dev[t], y, mode=mode)
            torch.cuda.synchronize()
            run.append((y, *ctx.last_routing()))
        outs.append((run, pred.stats()))
        ctx.close()
        pred.close()
    ws = torch.empty(S.route_workspace_bytes(cfg.B, cfg.E), dtype=torch.uint8, device=DEV)
    idx = torch.empty((cfg.B, cfg.K), dtype=torch.int32, device=DEV)
    w, z = torch.empty((cfg.B, cfg.K), device=DEV), torch.empty((cfg.B, cfg.E), device=DEV)
    for t in range(cfg.T):
        for l in range(cfg.L):
            S.route_topk(st.x_dev[t][l], st.wg_dev[l], cfg.K, idx, w, ws, logits=z)
            S.route_scored(z, cfg.K, idx, w, score=score, bias=bias[l].contiguous(), n_groups=groups, top_groups=top,
                           renorm=renorm, scale=1.5)
            ri, rw, _ = scoredref.route(z.cpu().numpy().astype(np.float64), cfg.K, score,
                                        bias[l].cpu().numpy().astype(np.float64), groups, top, 2, renorm, 1.5)
            ref = moe_ffn(decode_storage(st.x_store[t][l]), ri, rw, lambda e: expert_f64(cfg, l, e),
                          shared=[expert_f64(cfg, l, s, shared=True) for s in range(cfg.n_shared)])
            for run, stats in outs:
                y, i, ww = run[t]
                assert np.array_equal(i[l], ri) and np.array_equal(ww[l], w.cpu().numpy())
                assert np.linalg.norm(y[l].cpu().numpy() - ref) <= 1e-2 * np.linalg.norm(ref)
    for run, stats in outs[1:]:
        if mode:
            assert np.array_equal(stats, outs[0][1])


def test_few_candidates_and_return_to_the_plain_router():
    """All but one expert ruled out: the others come with weight 0, distinct; then the plain router again, in a replayed
    graph too."""
    import torch
    from paper_2606_15453_amd import stmoe as S
    from paper_2606_15453_amd import workload as W
    st = Stack(W.CONFIGS["tiny"].scaled(P=8, T=4, B=2, E=8, K=4, C=5))
    cfg = st.cfg
    bias = torch.full((cfg.L, cfg.E), -float("inf"), device=DEV)
    bias[:, 5] = 0.0
    plain, _, keep0 = _context(st, 0, 0, 0, False)
    for graph in (0, 1):
        ctx, _, keep = _context(st, 0, 0, graph, False)
        y, want = (torch.empty((cfg.L, cfg.B, cfg.H), device=DEV) for _ in range(2))
        for t in range(2):
            ctx.set_routing("sigmoid", bias)
            ctx.token(t, st.x_dev[t], y, mode=S.MODE_ON_DEMAND)
            idx, w = ctx.last_routing()
            assert (idx == np.array([5, 0, 1, 2])).all() and (w[..., 0] > 0).all() and not w[..., 1:].any()
            ctx.set_routing()
            ctx.token(t, st.x_dev[t], y, mode=S.MODE_ON_DEMAND)
            plain.token(t, st.x_dev[t], want, mode=S.MODE_ON_DEMAND)
            torch.cuda.synchronize()
            assert torch.equal(y, want) and np.array_equal(ctx.last_routing()[0], plain.last_routing()[0])
        for bad in (dict(score="sigmoid", n_groups=3), dict(score="sigmoid", n_groups=4, top_groups=1),
                    dict(score="sigmoid", n_groups=2, top_groups=3), dict(score="sigmoid", scale=float("nan")),
                    dict(score="sigmoid", group_top=3)):
            with pytest.raises(S.StmoeError):
                ctx.set_routing(**bad)
        with pytest.raises(ValueError):
            ctx.set_routing("sigmoid", bias[0])
        ctx.close()
