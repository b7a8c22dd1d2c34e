"""Timed cases of the scored router and of low-rank adapters.

route: softmax or sigmoid scores of logits, a bias for balance, the best groups of experts, the
top K in them and their weights; where `step` is set, the selections per expert and the bias's
step too.  route_grad: the gradient of those weights with respect to the logits.  lora: the
low-rank adapters of many requests added to a projection's result.  lora_grad: their gradient.

    listed()            the cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program has on the GPU before the call
    run(state)          one pass; returns every output: in plain torch, or with `own` by the
                        public binding (paper_2606_15453_amd.stmoe)
    work(case)          bytes and operations one pass cannot do without
    exact(case, seed)   what run() returns, in 64 bits
"""
import torch

own = False           # True: run() calls the framework's operators

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
RATE = 1e-3           # one step of the balance bias


def _route(name, kind, T, E, K, dtype, score, groups, top_groups, group_top=2, bias=True, renorm=True, scale=1.0,
           mask=False, step=False, ld=0):
    return dict(name=name, kind=kind, T=T, E=E, K=K, dtype=dtype, score=score, groups=groups, top_groups=top_groups,
                group_top=group_top, bias=bias, renorm=renorm, scale=scale, mask=mask, step=step, ld=ld or E)


def _lora(name, kind, T, Hin, Hout, n, R, dtype="bf16", y="bf16", mixed=False, ranks=False):
    return dict(name=name, kind=kind, T=T, Hin=Hin, Hout=Hout, n=n, R=R, dtype=dtype, y=y, mixed=mixed, ranks=ranks)


def listed():
    return [
        # one decode token of one user: launches and latency are all there is
        _route("route_t1_e128_f32", "route", 1, 128, 8, "f32", "sigmoid", 8, 4, scale=2.5),
        # sixteen users, softmax scores without a bias, a group as good as its best expert
        _route("route_t16_e64_bf16", "route", 16, 64, 6, "bf16", "softmax", 8, 3, group_top=1, bias=False, renorm=False),
        # a small training batch with padding, groups of twelve, rows inside a wider matrix
        _route("route_t1000_e60_bf16", "route", 1000, 60, 4, "bf16", "softmax", 5, 2, renorm=False, mask=True, step=True,
               ld=64),
        # a large training batch, sigmoid scores, half of eight groups
        _route("route_t32768_e256_f32", "route", 32768, 256, 8, "f32", "sigmoid", 8, 4, scale=2.5, step=True),
        # their gradients
        _route("route_grad_t1000_e60_bf16", "route_grad", 1000, 60, 4, "bf16", "softmax", 5, 2, renorm=False, mask=True,
               ld=64),
        _route("route_grad_t32768_e256_f32", "route_grad", 32768, 256, 8, "f32", "sigmoid", 8, 4, scale=2.5),
        # one decode token beside the expert block, whose result is fp32
        _lora("lora_t1_h2048_r16", "lora", 1, 2048, 2048, 8, 16, y="f32"),
        # a decode step of 64 users with adapters of several ranks, every row another adapter
        _lora("lora_t64_h4096_r64", "lora", 64, 4096, 4096, 32, 64, mixed=True, ranks=True),
        # the prompts of some requests, one after the other
        _lora("lora_t8192_h4096_r64", "lora", 8192, 4096, 4096, 8, 64),
        # beside a router of 61 experts, in fp32, at sizes that nothing divides
        _lora("lora_f32_t37_odd", "lora", 37, 1000, 61, 5, 12, dtype="f32", y="f32", mixed=True),
        # training steps: a small one in fp32, and one of four adapters at once
        _lora("lora_grad_f32_t300_odd", "lora_grad", 300, 520, 1000, 3, 12, dtype="f32", y="f32", mixed=True, ranks=True),
        _lora("lora_grad_t4096_h4096_r16", "lora_grad", 4096, 4096, 4096, 4, 16),
    ]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def draw(rng):
    """Routers over 1 to 32768 tokens and 2 to 256 experts in 1 to 16 groups; 1 to 8192 tokens
    with 1 to 64 adapters of rank 1 to 128 beside projections of 64 to 4096 columns in and 8 to
    4096 out."""
    kind = rng.choice(["route", "route", "route_grad", "lora", "lora", "lora_grad"])
    if kind.startswith("route"):
        G = rng.choice([1, 1, 2, 3, 4, 5, 8, 16])
        E = G * max(2, int(_log(rng, 2, 257)) // G)
        top = rng.randint(max(1, G // 4), G)
        K = rng.randint(1, min(10, E // G * top))
        T = max(1, min(int(_log(rng, 1, 32769)), 32768 * 256 // E))
        return dict(kind=kind, T=T, E=E, K=K, dtype=rng.choice(["bf16", "f32"]), score=rng.choice(["sigmoid", "softmax"]),
                    groups=G, top_groups=top, group_top=rng.choice([1, 2]), bias=rng.random() < 0.7,
                    renorm=rng.random() < 0.5, scale=rng.choice([1.0, 2.5]), mask=rng.random() < 0.5,
                    step=kind == "route" and rng.random() < 0.5, ld=E + rng.choice([0, 0, 1, 8]))
    Hin, Hout = int(_log(rng, 64, 4097)), int(_log(rng, 8, 4097))
    if rng.random() < 0.7:
        m = rng.choice([8, 64, 128])
        Hin, Hout = max(m, Hin // m * m), max(m, Hout // m * m)
    R = rng.choice([1, 4, 8, 8, 16, 16, 32, 64, 128, rng.randint(2, 100)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    y = dtype if kind == "lora_grad" else rng.choice(["bf16", "f32"])
    # of what the largest listed cases move and compute
    most_t, most_r = (8192, 64) if kind == "lora" else (4096, 16)
    T = int(_log(rng, 1, most_t + 1))
    while T > 1 and T * (Hin + Hout) * max(R, most_r) * (1 if dtype == y == "bf16" else 2) > most_t * 8192 * most_r:
        T = T * 2 // 3
    n = min(int(_log(rng, 1, 65)), max(1, 2 ** 23 // (R * (Hin + Hout))))
    return dict(kind=kind, T=T, Hin=Hin, Hout=Hout, n=n, R=R, dtype=dtype, y=y, mixed=rng.random() < 0.5,
                ranks=rng.random() < 0.3)


# ------------------------------------------------------------------ inputs
def _gen(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + what)
    return g


def _randn(shape, seed, what, scale=1.0):
    return torch.randn(shape, generator=_gen(seed, what), device=DEV) * scale


def _prepare_route(case, seed):
    st = dict(case=case)
    T, E, K = case["T"], case["E"], case["K"]
    # tokens differ, and experts in popularity
    z = 1.5 * _randn((T, case["ld"]), seed, 1) + 0.5 * _randn((1, case["ld"]), seed, 2)
    st["logits"] = z.to(DT[case["dtype"]])[:, :E]
    # some tens of steps either way, as a while of training leaves it
    steps = torch.randint(-60, 61, (E,), generator=_gen(seed, 3), device=DEV)
    top = 1.0 if case["score"] == "sigmoid" else 2.0 / E
    st["bias"] = steps * (RATE * top) if case["bias"] else None
    st["mask"] = None
    if case["mask"]:      # padding at the end of sequences: about one token in twelve
        st["mask"] = (torch.rand(T, generator=_gen(seed, 4), device=DEV) >= 0.08).to(torch.uint8)
    if case["kind"] == "route_grad":
        st.update(idx=_route_plain(st)[0], d_w=_randn((T, K), seed, 5, 1e-3))
        if own:
            st["d_logits"] = torch.empty((T, E), dtype=DT[case["dtype"]], device=DEV)
    elif own:
        st["idx"] = torch.empty((T, K), dtype=torch.int32, device=DEV)
        st["w"] = torch.empty((T, K), device=DEV)
        if case["step"]:
            st["counts"] = torch.empty(E, dtype=torch.int32, device=DEV)
            st["new_bias"] = torch.empty(E, device=DEV)
    if case["step"] and not case["bias"]:
        st["old_bias"] = torch.zeros(E, device=DEV)
    return st


def _prepare_lora(case, seed):
    st = dict(case=case)
    T, Hin, Hout, n, R = (case[k] for k in ("T", "Hin", "Hout", "n", "R"))
    dt, ydt, grad = DT[case["dtype"]], DT[case["y"]], case["kind"] == "lora_grad"
    st["x"] = _randn((T, Hin), seed, 1).to(dt)
    st["base"] = _randn((T, Hin if grad else Hout), seed, 2).to(ydt)
    # a decode step's rows go by the users, a prompt's tokens stand together; one in sixteen has no adapter
    runs = T if case["mixed"] else min(T, 2 * n)
    of_run = torch.randint(0, n, (runs,), generator=_gen(seed, 3), device=DEV)
    of_run[torch.rand(runs, generator=_gen(seed, 4), device=DEV) < 1 / 16] = -1
    ends = torch.rand(runs, generator=_gen(seed, 5), device=DEV) + 0.25
    ends = (ends.cumsum(0) / ends.sum() * T).long()
    run_of = torch.arange(T, device=DEV) if case["mixed"] else torch.searchsorted(ends, torch.arange(T, device=DEV), right=True)
    st["adapter"] = of_run[run_of.clamp(max=runs - 1)].to(torch.int32)
    ranks = torch.full((n,), R, dtype=torch.int32, device=DEV)
    if case["ranks"]:     # an adapter has its whole rank, half or a quarter of it
        ranks = (ranks >> torch.randint(0, 3, (n,), generator=_gen(seed, 6), device=DEV, dtype=torch.int32)).clamp(min=1)
    st["ranks"] = ranks if case["ranks"] else None
    inside = (torch.arange(R, device=DEV) < ranks[:, None])[:, :, None]
    st["a"] = (_randn((n, R, Hin), seed, 7, Hin ** -0.5) * inside).to(dt)
    st["b"] = (_randn((n, R, Hout), seed, 8, 0.3 * R ** -0.5) * inside).to(dt)
    st["scales"] = 0.5 + 1.5 * torch.rand(n, generator=_gen(seed, 9), device=DEV)
    if grad:
        st["dy"] = _randn((T, Hout), seed, 10, 1e-2).to(dt)
        st["v"] = _by_adapter(st, lambda x, a: torch.bmm(x, a.transpose(1, 2).contiguous()), st["x"], st["a"])
    if own:
        from paper_2606_15453_amd import stmoe as S
        at = lambda t: torch.tensor([m.data_ptr() for m in t], dtype=torch.int64, device=DEV)
        st["a_ptrs"], st["b_ptrs"] = at(st["a"]), at(st["b"])
        st["plan"] = torch.empty(S.lora_plan_bytes(T, n), dtype=torch.uint8, device=DEV)
        S.lora_plan(st["adapter"], n, st["plan"])
        bytes_of = S.lora_backward_workspace_bytes if grad else S.lora_workspace_bytes
        st["ws"] = torch.empty(bytes_of(T, Hin, Hout, n, R, dt), dtype=torch.uint8, device=DEV)
        st["y"] = torch.empty_like(st["base"])
        if grad:
            st["da"], st["db"] = torch.zeros((n, R, Hin), device=DEV), torch.zeros((n, R, Hout), device=DEV)
            st["da_ptrs"], st["db_ptrs"] = at(st["da"]), at(st["db"])
    return st


def prepare(case, seed):
    return _prepare_route(case, seed) if case["kind"].startswith("route") else _prepare_lora(case, seed)


# ------------------------------------------------------------------ plain forms
def _scores(z, score):
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    ex = torch.exp(z - z.amax(dim=1, keepdim=True))
    return ex / ex.sum(dim=1, keepdim=True)


def _route_plain(st):
    """Selection and weights (a choice between near scores needs their 64 bits)."""
    c = st["case"]
    T, E, K, G = c["T"], c["E"], c["K"], c["groups"]
    z = st["logits"].double()
    s = _scores(z, c["score"])
    choice = z if st["bias"] is None else s + st["bias"].double()
    if c["top_groups"] < G:
        of = (choice if c["group_top"] == 1 or st["bias"] is not None else s).view(T, G, E // G)
        best = of.sort(dim=2, descending=True)[0][:, :, :c["group_top"]].sum(dim=2)
        kept = best.sort(dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        allowed = (kept[:, :, None] == torch.arange(G, device=z.device)).any(dim=1)
        choice = torch.where(allowed.repeat_interleave(E // G, dim=1), choice, -torch.inf)
    idx = choice.sort(dim=1, descending=True, stable=True)[1][:, :K]
    w = s.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    w, idx = (w * c["scale"]).float(), idx.to(torch.int32)
    if st["mask"] is not None:
        live = st["mask"][:, None] != 0
        w, idx = torch.where(live, w, 0.0), torch.where(live, idx, -1)
    return idx, w


def _bias_step(st, idx):
    E = st["case"]["E"]
    counts = (idx.flatten()[:, None] == torch.arange(E, device=idx.device)).sum(dim=0)
    old = st["bias"] if st["bias"] is not None else st["old_bias"]
    return counts.to(torch.int32), old + RATE * torch.sign(counts.sum() - E * counts).float()


def _route_grad_plain(st):
    c = st["case"]
    z, idx = st["logits"].float(), st["idx"].long()
    live, at = idx[:, :1] >= 0, idx.clamp(min=0)
    s = _scores(z, c["score"])
    sel, g = s.gather(1, at), c["scale"] * st["d_w"]
    if c["renorm"]:
        total = sel.sum(dim=1, keepdim=True)
        q = sel / total
        g = (g - (q * g).sum(dim=1, keepdim=True)) / total
    if c["score"] == "sigmoid":
        rest = 1 / (1 + torch.exp(z.gather(1, at)))
        d_z = torch.zeros_like(z).scatter_add(1, at, g * sel * rest)
    else:
        d_z = torch.zeros_like(z).scatter_add(1, at, g * sel) - s * (g * sel).sum(dim=1, keepdim=True)
    return torch.where(live, d_z, 0.0).to(DT[c["dtype"]])


def _by_adapter(st, f, *rows_and_matrices):
    """f over the tokens of each adapter, padded to the most that one has: rows [T][...] become
    [n][most][...]; matrices [n][...] stay.  f's rows return to their tokens (0 without an adapter)."""
    n, T = st["case"]["n"], st["case"]["T"]
    a, order = st["adapter"].long().sort(stable=True)
    order, a = order[a >= 0], a[a >= 0]
    count = (a[:, None] == torch.arange(n, device=a.device)).sum(dim=0)
    pos = torch.arange(len(a), device=a.device) - (count.cumsum(0) - count)[a]

    def padded(m):
        if m.shape[0] == n and m.dim() == 3:
            return m.float()
        out = torch.zeros((n, max(1, int(count.max())), m.shape[1]), device=m.device)
        out[a, pos] = m[order].float()
        return out

    got = f(*(padded(m) for m in rows_and_matrices))
    out = torch.zeros((T, got.shape[2]), device=got.device)
    out[order] = got[a, pos]
    return out


def _lora_plain(st):
    scale = st["scales"][:, None, None]
    delta = _by_adapter(st, lambda x, a, b: torch.bmm(torch.bmm(x, a.transpose(1, 2).contiguous()) * scale, b),
                        st["x"], st["a"], st["b"])
    return (st["base"].float() + delta).to(DT[st["case"]["y"]])


def _lora_grad_plain(st):
    scale, grads = st["scales"][:, None, None], []

    def f(x, dy, v, a, b):
        u = torch.bmm(dy, b.transpose(1, 2).contiguous()) * scale
        grads.append(torch.bmm(u.transpose(1, 2).contiguous(), x))
        grads.append(torch.bmm(v.transpose(1, 2).contiguous(), dy) * scale)
        return torch.bmm(u, a)

    dx = _by_adapter(st, f, st["x"], st["dy"], st["v"], st["a"], st["b"])
    if st["ranks"] is not None:
        inside = torch.arange(st["case"]["R"], device=DEV) < st["ranks"][:, None]
        grads = [torch.where(inside[:, :, None], m, 0.0) for m in grads]
    return (st["base"].float() + dx).to(DT[st["case"]["y"]]), grads[0], grads[1]


def run(st):
    c = st["case"]
    if own:
        from paper_2606_15453_amd import stmoe as S
        if c["kind"] == "route":
            counts = st["counts"].zero_() if c["step"] else None
            S.route_scored(st["logits"], c["K"], st["idx"], st["w"], score=c["score"], bias=st["bias"],
                           n_groups=c["groups"], top_groups=c["top_groups"], group_top=c["group_top"],
                           renorm=c["renorm"], scale=c["scale"], mask=st["mask"], counts=counts)
            if not c["step"]:
                return st["idx"], st["w"]
            old = st["bias"] if st["bias"] is not None else st["old_bias"]
            S.route_bias_step(counts, old, RATE, out=st["new_bias"])
            return st["idx"], st["w"], counts, st["new_bias"]
        if c["kind"] == "route_grad":
            S.route_scored_backward(st["logits"], st["idx"], st["d_w"], st["d_logits"], score=c["score"],
                                    renorm=c["renorm"], scale=c["scale"])
            return st["d_logits"]
        if c["kind"] == "lora":
            S.lora(st["x"], st["plan"], st["a_ptrs"], st["b_ptrs"], c["R"], st["y"], st["ws"], base=st["base"],
                   ranks=st["ranks"], scales=st["scales"])
            return st["y"]
        S.lora_backward(st["x"], st["dy"], st["v"], st["plan"], st["a_ptrs"], st["b_ptrs"], c["R"], st["da_ptrs"],
                        st["db_ptrs"], st["ws"], dx=st["y"], base=st["base"], ranks=st["ranks"], scales=st["scales"])
        return st["y"], st["da"], st["db"]
    if c["kind"] == "route":
        idx, w = _route_plain(st)
        return (idx, w, *_bias_step(st, idx)) if c["step"] else (idx, w)
    if c["kind"] == "route_grad":
        return _route_grad_plain(st)
    return _lora_plain(st) if c["kind"] == "lora" else _lora_grad_plain(st)


# ------------------------------------------------------------------ work
def work(case):
    if case["kind"].startswith("route"):
        T, E, K, size = case["T"], case["E"], case["K"], SIZE[case["dtype"]]
        if case["kind"] == "route":
            return {"bytes": T * (E * size + 8 * K + int(case["mask"])) + 4 * E * (1 + 2 * int(case["step"])),
                    "flops": 8 * T * E}
        # of the logits the selected ones alone, where no other score matters
        read = E if case["score"] == "softmax" and not case["renorm"] else K
        return {"bytes": T * (E * size + read * size + 8 * K), "flops": 4 * T * read}
    T, Hin, Hout, n, R = (case[k] for k in ("T", "Hin", "Hout", "n", "R"))
    size, ysize = SIZE[case["dtype"]], SIZE[case["y"]]
    rank = R * 7 / 12 if case["ranks"] else R
    used = n * (1 - (1 - 1 / n) ** (T if case["mixed"] else min(T, 2 * n)))
    if case["kind"] == "lora":
        return {"bytes": int(T * (Hin * size + 2 * Hout * ysize + 4) + used * rank * (Hin + Hout) * size),
                "flops": int(2 * T * rank * (Hin + Hout))}
    return {"bytes": int(T * (Hin * size + Hout * size + 2 * Hin * ysize + 4 * rank + 4)
                         + rank * (Hin + Hout) * (used * size + 4 * n)),
            "flops": int(4 * T * rank * (Hin + Hout))}


# ------------------------------------------------------------------ exact
def _exact_route(st):
    c = st["case"]
    T, E, K, G = c["T"], c["E"], c["K"], c["groups"]
    z = st["logits"].double()
    s = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z, dim=1)
    value = s if st["bias"] is None else s + st["bias"].double()
    left = z.clone() if st["bias"] is None else value.clone()
    rows = torch.arange(T, device=DEV)

    def first_best(m):      # the first of the largest ones
        return (m == m.amax(dim=1, keepdim=True)).to(torch.uint8).argmax(dim=1)

    if c["top_groups"] < G:
        by = (left if c["group_top"] == 1 else value).clone().view(T, G, E // G)
        best = by.amax(dim=2)
        if c["group_top"] == 2:
            at = by.argmax(dim=2, keepdim=True)
            best = best + by.scatter(2, at, -torch.inf).amax(dim=2)
        out = torch.ones((T, G), dtype=torch.bool, device=DEV)
        for _ in range(c["top_groups"]):
            g = first_best(best)
            out[rows, g] = False
            best[rows, g] = -torch.inf
        left.view(T, G, E // G)[out] = -torch.inf
    idx = torch.empty((T, K), dtype=torch.int64, device=DEV)
    for k in range(K):
        idx[:, k] = first_best(left)
        left[rows, idx[:, k]] = -torch.inf
    w = torch.gather(s, 1, idx)
    if c["renorm"]:
        w /= w.sum(dim=1, keepdim=True)
    w *= c["scale"]
    if st["mask"] is not None:
        idx[st["mask"] == 0], w[st["mask"] == 0] = -1, 0
    out = (idx.to(torch.int32), w)
    if c["step"]:
        counts = torch.bincount(idx[idx >= 0], minlength=E)
        old = torch.zeros(E, dtype=torch.float64, device=DEV) if st["bias"] is None else st["bias"].double()
        load = counts.double() - counts.double().mean()
        load[(counts * E) == counts.sum()] = 0
        out += (counts.to(torch.int32), old - RATE * torch.sign(load))
    return out


def _exact_route_grad(st):
    c, z = st["case"], st["logits"].double().requires_grad_(True)
    s = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z, dim=1)
    live = st["idx"][:, 0] >= 0
    w = s[live].gather(1, st["idx"][live].long())
    if c["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    return torch.autograd.grad((w * st["d_w"][live].double()).sum() * c["scale"], z)[0]


def _exact_lora(st):
    c, y = st["case"], st["base"].double()
    for i in range(c["n"]):
        rows = (st["adapter"] == i).nonzero().squeeze(1)
        if len(rows):
            A, B = st["a"][i].double(), st["b"][i].double()
            y[rows] += st["scales"][i].double() * ((st["x"][rows].double() @ A.T) @ B)
    return y


def _exact_lora_grad(st):
    c, dx = st["case"], st["base"].double()
    da = torch.zeros((c["n"], c["R"], c["Hin"]), dtype=torch.float64, device=DEV)
    db = torch.zeros((c["n"], c["R"], c["Hout"]), dtype=torch.float64, device=DEV)
    for i in range(c["n"]):
        rows = (st["adapter"] == i).nonzero().squeeze(1)
        if not len(rows):
            continue
        r = c["R"] if st["ranks"] is None else int(st["ranks"][i])
        A, B, s = st["a"][i, :r].double(), st["b"][i, :r].double(), st["scales"][i].double()
        x, dy, v = st["x"][rows].double(), st["dy"][rows].double(), st["v"][rows, :r].double()
        u = s * (dy @ B.T)
        da[i, :r], db[i, :r] = u.T @ x, s * (v.T @ dy)
        dx[rows] += u @ A
    return dx, da, db


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    return {"route": _exact_route, "route_grad": _exact_route_grad, "lora": _exact_lora,
            "lora_grad": _exact_lora_grad}[case["kind"]](st)
