"""The mixture-of-experts operators in 64 bits, one token at a time, straight from their definitions."""
import numpy as np

INF = float("inf")


def scores(l, score):
    """l: logits of one token in float64. Experts at -inf or NaN have score 0."""
    live = l > -INF
    s = np.zeros(l.shape)
    if not live.any():
        return s
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            s[live] = 1.0 / (1.0 + np.exp(-l[live]))
        return s
    m = l[live].max()
    s[live] = [1.0 if v == m else np.exp(v - m) for v in l[live]]
    return s / s.sum()


def route(logits, top_k, score="softmax", bias=None, mask=None, groups=1, top_groups=1, group_top=1, renormalize=False,
          scale=1.0, **_):
    """Choices and weights, and for every token the least distance between values whose order decides a choice."""
    T, E = logits.shape
    index, weight, margin = np.full((T, top_k), -1), np.zeros((T, top_k)), np.full(T, INF)
    for t in range(T):
        l = logits[t]
        s = scores(l, score)
        live = l > -INF
        by_score = np.where(live, s + (bias if bias is not None else 0.0), -INF)
        choice = by_score.copy() if bias is not None else np.where(live, l, -INF)
        choice[~(choice > -INF)] = -INF
        by_score[~(by_score > -INF)] = -INF
        if top_groups < groups:
            value = []
            for g in range(groups):
                part = np.sort((by_score if group_top == 2 else choice).reshape(groups, -1)[g])[::-1]
                part = part[part > -INF][:group_top]
                value.append(part.sum() if part.size else -INF)
            value = np.array(value)
            order = np.argsort(-value, kind="stable")
            if (group_top == 2 or bias is not None) and value[order[top_groups - 1]] > -INF:
                margin[t] = value[order[top_groups - 1]] - value[order[top_groups]]
            closed = [g for g in order[top_groups:]] + [g for g in range(groups) if value[g] == -INF]
            for g in closed:
                choice.reshape(groups, -1)[g] = -INF
        order = np.argsort(-choice, kind="stable")
        if bias is not None:
            top = choice[order][:top_k + 1]
            top = top[top > -INF]
            if top.size > 1:
                margin[t] = min(margin[t], (top[:-1] - top[1:]).min())
        if mask is not None and not mask[t]:
            continue
        index[t] = [e if choice[e] > -INF else -1 for e in order[:top_k]]
        u = np.array([s[e] if e >= 0 else 0.0 for e in index[t]])
        if renormalize:
            u = u / u.sum() if u.sum() > 0 else 0.0 * u
        weight[t] = u * scale
    return index, weight, margin


def weights_of(l, chosen, score, renormalize, scale):
    """The weights of given choices as a function of one token's logits."""
    s = scores(l, score)
    u = np.array([s[e] if e >= 0 else 0.0 for e in chosen])
    if renormalize:
        u = u / u.sum() if u.sum() > 0 else 0.0 * u
    return u * scale


def route_backward(logits, index, grad, score="softmax", renormalize=False, scale=1.0, **_):
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        s = scores(logits[t], score)
        some = (index[t] >= 0) & (index[t] < E)
        at = np.where(some, index[t], 0)
        u, g = np.where(some, s[at], 0.0), np.where(some, grad[t], 0.0) * scale
        du = g
        if renormalize:
            r = u.sum()
            du = np.where(some, (g - (g * u).sum() / r) / r, 0.0) if r > 0 else 0.0 * g
        ds = np.zeros(E)
        np.add.at(ds, at[some], du[some])
        out[t] = s * (ds - (ds * s).sum()) if score == "softmax" else ds * s * (1.0 - s)
    return out


def plan(index, experts, capacity):
    flat = index.reshape(-1)
    row, nxt, offsets = np.full(flat.size, -1), 0, [0]
    for e in range(experts):
        for i in np.nonzero(flat == e)[0]:
            row[i] = nxt if nxt < capacity else -1
            nxt += 1
        offsets.append(min(nxt, capacity))
    return row.reshape(index.shape), np.array(offsets)


def dispatch(x, row, out):
    out = out.copy()
    for t in range(row.shape[0]):
        for r in row[t]:
            if 0 <= r < out.shape[0]:
                out[r] = x[t]
    return out


def combine(z, row, weight):
    """The sums, and the sums of their terms' magnitudes."""
    y = np.zeros((row.shape[0], z.shape[1]))
    size = y.copy()
    for t in range(row.shape[0]):
        for k, r in enumerate(row[t]):
            if 0 <= r < z.shape[0]:
                w = 1.0 if weight is None else weight[t, k]
                y[t] += w * z[r]
                size[t] += np.abs(w * z[r])
    return y, size


def combine_backward(grad, z, row, weight, grad_z):
    grad_z, dw, size = grad_z.copy(), np.zeros(row.shape), np.zeros(row.shape)
    for t in range(row.shape[0]):
        for k, r in enumerate(row[t]):
            if 0 <= r < z.shape[0]:
                grad_z[r] = weight[t, k] * grad[t]
                dw[t, k] = (grad[t] * z[r]).sum()
                size[t, k] = np.abs(grad[t] * z[r]).sum()
    return grad_z, dw, size


def silu_gate(x):
    g, u = np.split(x.astype(np.float64), 2, axis=1)
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * u


def quantize(x):
    """Codes and scales of rows held in 32 bits; the reciprocal and the products are rounded to 32 bits."""
    x = x.astype(np.float32)
    codes, scale = np.zeros(x.shape, np.int8), np.zeros(x.shape[0], np.float32)
    for i in range(x.shape[0]):
        m = np.abs(x[i]).max() if x.shape[1] else np.float32(0)
        if not np.isfinite(m):
            scale[i] = m
        elif m >= np.float32(2.0 ** -119):
            codes[i] = np.rint(x[i] * (np.float32(1) / m * np.float32(127))).astype(np.int8)
            scale[i] = m / np.float32(127)
    return codes, scale


def product(codes, scale, weights, weight_scale, offsets, out):
    out = out.copy()
    E = weights.shape[0]
    R = codes.shape[0]
    ends = [0, R] if offsets is None else offsets
    for s in range(len(ends) - 1):
        a, b = min(max(ends[s], 0), R), min(max(ends[s + 1], 0), R)
        if b > a:
            sums = codes[a:b].astype(np.float64) @ weights[s % E].astype(np.float64).T  # whole numbers below 2^53
            out[a:b] = sums * scale[a:b, None].astype(np.float64) * weight_scale[s % E].astype(np.float64)
    return out
