"""Plain 64-bit forms of the 4-bit expert operators and of the balanced router
(numpy; nothing of the library is used)."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)


def mx_quantize(x):
    """(codes [r][ceil(c/2)], scales [r][ceil(c/32)], values [r][c]) of x, one element at a time by its distance to
    every magnitude (ties: the even code)."""
    x = np.asarray(x, np.float64)
    r, c = x.shape
    nb = -(-c // 32)
    codes = np.zeros((r, nb * 32), np.uint8)
    scales = np.zeros((r, nb), np.uint8)
    values = np.zeros((r, c))
    for b in range(nb):
        v = x[:, 32 * b:32 * b + 32]
        n = v.shape[1]
        bad = ~np.isfinite(v).all(axis=1)
        v = np.where(bad[:, None], 0.0, v)
        top = np.abs(v).max(axis=1)
        e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1 - 2, -127)
        e = np.maximum(e, -127)
        far = np.abs(np.abs(v)[:, :, None] / np.exp2(e.astype(np.float64))[:, None, None] - GRID)
        code = far.argmin(axis=2)
        up = np.minimum(code + 1, 7)
        tie = (np.take_along_axis(far, up[..., None], 2) == np.take_along_axis(far, code[..., None], 2))[..., 0]
        code = np.where(tie & (code % 2 == 1) & (up > code), up, code)
        val = GRID[code] * np.exp2(e.astype(np.float64))[:, None] * np.where(np.signbit(v), -1, 1)
        code = code + 8 * np.signbit(v)
        codes[:, 32 * b:32 * b + n] = np.where(bad[:, None], 0, code)
        scales[:, b] = np.where(bad, 255, e + 127)
        values[:, 32 * b:32 * b + n] = np.where(bad[:, None], np.nan, val)
    half = -(-c // 2)
    packed = codes[:, 0:2 * half:2] | (codes[:, 1:2 * half + 1:2][:, :half] << 4)
    return packed, scales, values


def mx_values(codes, scales, cols):
    """Values of codes [..][ceil(c/2)] and scales [..][ceil(c/32)]."""
    both = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)[..., :cols]
    e = np.repeat(scales.astype(np.float64) - 127, 32, axis=-1)[..., :cols]
    v = np.where(both < 8, 1, -1) * GRID[both & 7] * np.exp2(e)
    return np.where(np.repeat(scales, 32, axis=-1)[..., :cols] == 255, np.nan, v)


def moe_ffn(x, idx, w, experts, shared=()):
    """y [T][H]: experts[e] = (gate, up, down) values; entries outside the experts and repeats are ignored."""
    x = np.asarray(x, np.float64)
    y = np.zeros_like(x)

    def add(rows, wt, mats):
        g, u = x[rows] @ mats[0].T, x[rows] @ mats[1].T
        with np.errstate(over="ignore", invalid="ignore"):
            y[rows] += wt[:, None] * ((g / (1 + np.exp(-g)) * u) @ mats[2].T)

    first = np.ones(idx.shape, bool)
    for k in range(1, idx.shape[1]):
        first[:, k] = ~(idx[:, :k] == idx[:, k:k + 1]).any(axis=1)
    for e in range(len(experts)):
        hit = (idx == e) & first
        rows = np.nonzero(hit.any(axis=1))[0]
        if len(rows):
            add(rows, (np.where(hit, w, 0).sum(axis=1))[rows], experts[e])
    for m in shared:
        add(np.arange(len(x)), np.ones(len(x)), m)
    return y


def balance(z, K, renorm=False, mask=None):
    """dict of idx, w, counts, n, prob_sum, loss (balance, z) of logits z [T][E]."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    cand = z != -np.inf
    live = cand.any(axis=1) & (np.ones(T, bool) if mask is None else np.asarray(mask) != 0)
    idx, w = np.full((T, K), -1, np.int32), np.zeros((T, K))
    prob, lse = np.zeros((T, E)), np.zeros(T)
    for t in np.nonzero(live)[0]:
        order = sorted(np.nonzero(cand[t])[0], key=lambda e: (np.isnan(z[t, e]), -z[t, e] if z[t, e] == z[t, e] else 0, e))
        pick = order[:K]
        top = z[t, order[0]]
        ex = np.where(cand[t], np.exp(z[t] - top), 0.0)
        prob[t] = ex / ex.sum()
        lse[t] = top + np.log(ex.sum())
        idx[t, :len(pick)] = pick
        w[t, :len(pick)] = ex[pick] / (ex[pick].sum() if renorm else ex.sum())
    counts = np.bincount(idx[idx >= 0], minlength=E)
    n = int(live.sum())
    d = max(n, 1)
    loss = np.array([E * (counts / (d * K) * prob.sum(axis=0) / d).sum(), (lse ** 2).sum() / d])
    return dict(idx=idx, w=w, counts=counts, n=n, prob_sum=prob.sum(axis=0), loss=loss, prob=prob, lse=lse, live=live)


def balance_total(z, idx, counts, n, d_w, d_loss, renorm):
    """sum of d_w * gate weights and d_loss * losses as a function of z, selection and counts constant."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    K = idx.shape[1]
    live = idx[:, 0] >= 0
    d = max(n, 1)
    total = 0.0
    prob = np.zeros(E)
    for t in np.nonzero(live)[0]:
        top = z[t].max()
        ex = np.exp(z[t] - top)
        p = ex / ex.sum()
        prob += p
        total += d_loss[1] * (top + np.log(ex.sum())) ** 2 / d
        sel = idx[t][idx[t] >= 0]
        wt = p[sel] / p[sel].sum() if renorm else p[sel]
        total += (wt * d_w[t][idx[t] >= 0]).sum()
    return total + d_loss[0] * E * (counts / (d * K) * prob / d).sum()


def balance_grad(z, idx, counts, n, d_w, d_loss, renorm):
    """Its gradient, by the formula."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    K = idx.shape[1]
    d = max(n, 1)
    out = np.zeros((T, E))
    for t in np.nonzero(idx[:, 0] >= 0)[0]:
        top = z[t].max()
        ex = np.where(z[t] == -np.inf, 0.0, np.exp(z[t] - top))
        p, lse = ex / ex.sum(), top + np.log(ex.sum())
        a = d_loss[0] * E * counts / (d * d * K)
        ok = idx[t] >= 0
        sel, g = idx[t][ok], d_w[t][ok]
        if not renorm:
            a = a.copy()
            a[sel] += g
        out[t] = p * (a - (p * a).sum()) + 2 * d_loss[1] / d * lse * p
        if renorm:
            wt = p[sel] / p[sel].sum()
            out[t, sel] += wt * (g - (wt * g).sum())
    return out
