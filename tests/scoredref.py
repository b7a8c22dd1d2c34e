"""Plain 64-bit forms of routing by scores and of low-rank adapters (numpy; nothing
of the library is used)."""
import numpy as np


def scores(z, score):
    """Softmax or sigmoid of every row; minus infinity is no candidate and has 0."""
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if score == "sigmoid":
            return np.where(z == -np.inf, 0.0, 1 / (1 + np.exp(-z)))
        top = np.fmax.reduce(z, axis=1, keepdims=True)
        ex = np.where(z == -np.inf, 0.0, np.exp(z - top))
        return ex / ex.sum(axis=1, keepdims=True)


def _ranked(values, candidate):
    """Indices of the candidates, best first: numbers descending, then NaN; equal ones by index."""
    at = [i for i in range(len(values)) if candidate[i]]
    return sorted(at, key=lambda i: (np.isnan(values[i]), 0.0 if np.isnan(values[i]) else -values[i], i))


def route(z, K, score, bias=None, groups=1, top_groups=1, group_top=2, renorm=False, scale=1.0, mask=None):
    """(idx [T][K], w [T][K], counts [E])"""
    T, E = z.shape
    s = scores(z, score)
    idx, w = np.full((T, K), -1, np.int32), np.zeros((T, K))
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        cand = z[t] != -np.inf
        if bias is not None:
            cand &= bias != -np.inf
        value = s[t] if bias is None else s[t] + bias
        choice = z[t] if bias is None else value
        if top_groups < groups:
            size, best = E // groups, []
            by = choice if group_top == 1 else value
            for g in range(groups):
                r = _ranked(by[g * size:(g + 1) * size], cand[g * size:(g + 1) * size])[:group_top]
                best.append(sum((by[g * size + i] for i in r[1:]), by[g * size + r[0]]) if r else -np.inf)
            has = [cand[g * size:(g + 1) * size].any() for g in range(groups)]
            kept = _ranked(np.array(best), has)[:top_groups]
            cand = cand & np.isin(np.arange(E) // size, kept)
        sel = _ranked(choice, cand)[:K]
        idx[t, :len(sel)] = sel
        p = s[t][sel]
        if renorm and len(sel):
            zs = z[t][sel]
            with np.errstate(invalid="ignore", over="ignore"):
                # the ratios of the sigmoids also where they are below the smallest number
                p = np.exp(zs - zs.max()) if score == "sigmoid" and zs.max() < -64 else p
                p = p / p.sum()
        w[t, :len(sel)] = scale * p
    return idx, w, np.bincount(idx[idx >= 0], minlength=E)


def route_grad(z, idx, d_w, score, renorm, scale):
    """d_logits from the gradients of the weights, the selection a constant."""
    s, out = scores(z, score), np.zeros_like(z)
    for t in range(len(z)):
        k = idx[t] >= 0
        e, g = idx[t][k], scale * d_w[t][k]
        if not len(e):
            continue
        p = s[t][e]
        if renorm:
            zs = z[t][e]
            p = np.exp(zs - zs.max()) if score == "sigmoid" and zs.max() < -64 else p
            p = p / p.sum()
            g = g - (p * g).sum()
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                np.add.at(out[t], e, p * g / (1 + np.exp(z[t][e])))
        else:
            np.add.at(out[t], e, p * g)
            if not renorm:
                out[t] -= s[t] * (p * g).sum()
    return out


def bias_step(counts, bias, rate):
    counts = np.asarray(counts, np.int64)
    return bias + rate * np.sign(counts.sum(axis=-1, keepdims=True) - counts * counts.shape[-1])


def lora(x, adapter, A, B, scales, base):
    """(y [T][Hout], {token: v}) of lists of A [r][Hin] and B [r][Hout]; adapters outside the list: base alone."""
    y, v = np.array(base, np.float64), {}
    for a in range(len(A)):
        rows = np.flatnonzero(adapter == a)
        va = x[rows] @ A[a].T
        y[rows] += scales[a] * (va @ B[a])
        v.update(zip(rows, va))
    return y, v


def lora_grad(x, dy, adapter, A, B, scales, base):
    """(dx [T][Hin], [dA], [dB])"""
    dx, dA, dB = np.array(base, np.float64), [], []
    for a in range(len(A)):
        rows = np.flatnonzero(adapter == a)
        u = scales[a] * (dy[rows] @ B[a].T)
        dx[rows] += u @ A[a]
        dA.append(u.T @ x[rows])
        dB.append(scales[a] * ((x[rows] @ A[a].T).T @ dy[rows]))
    return dx, dA, dB
