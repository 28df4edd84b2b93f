"""Plain 64-bit implementations of the expert-layer operators (numpy, loops), written from their definitions."""
import numpy as np
import torch

EPS32 = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # relative, one rounding to nearest: 2^-p for p significant bits (24, 8, 11)
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # smallest step of the type


def route(logits, k, score, bias=None, mask=None, groups=1, top_groups=1, group_best=1, renorm=True, scale=1.0):
    """ids, weights, smallest nonzero distance between neighbouring keys or group scores that the choices hang on."""
    T, E = logits.shape
    ids, w = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    gap = np.inf
    bias_of = np.zeros(E) if bias is None else bias
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        x = logits[t].astype(np.float64)
        on = ~((x == -np.inf) | (bias_of == -np.inf))
        if np.isnan(x[on]).any() or np.isnan(bias_of[on]).any() or (bias_of[on] == np.inf).any() or (score == "softmax" and (x[on] == np.inf).any()):
            w[t] = np.nan
            continue
        s = np.zeros(E)
        with np.errstate(over="ignore"):
            if score == "sigmoid":
                s[on] = 1 / (1 + np.exp(-x[on]))
            elif on.any():
                e = np.exp(x[on] - x[on].max())
                s[on] = e / e.sum()
        key = x.copy() if (score == "softmax" and bias is None) else s + bias_of
        alive = on.copy()
        if groups > 1:
            per = E // groups
            gs = np.full(groups, -np.inf)
            for g in range(groups):
                ks = np.sort(key[g * per:(g + 1) * per][on[g * per:(g + 1) * per]])[::-1][:group_best]
                if ks.size:
                    gs[g] = ks.sum()
            order = np.argsort(-gs, kind="stable")
            d = -np.diff(gs[order][np.isfinite(gs[order])])
            if (d > 0).any():
                gap = min(gap, d[d > 0].min())
            keep = np.zeros(groups, dtype=bool)
            keep[order[:top_groups]] = True
            alive &= np.repeat(keep, per)
        where = np.nonzero(alive)[0]
        order = where[np.argsort(-key[where], kind="stable")]
        d = -np.diff(key[order[:k + 1]])
        if (d > 0).any():
            gap = min(gap, d[d > 0].min())
        n = min(k, order.size)
        ids[t, :n] = order[:n]
        c = s[order[:n]]
        if renorm:
            c = c / c.sum() if c.sum() > 0 else c
        w[t, :n] = c * scale
    return ids, w, gap


def layout(ids, E):
    """counts, offsets, slots, source: rows by expert, then by token."""
    flat = ids.reshape(-1)
    source = np.concatenate([np.nonzero(flat == e)[0] for e in range(E)] + [np.zeros(0, dtype=np.int64)])
    counts = np.array([(flat == e).sum() for e in range(E)], dtype=np.int64)
    slots = np.full(flat.size, -1, dtype=np.int64)
    slots[source] = np.arange(source.size)
    full = np.full(flat.size, -1, dtype=np.int64)
    full[: source.size] = source
    return counts, np.concatenate([[0], np.cumsum(counts)]), slots.reshape(ids.shape), full


def route_grad(logits, ids, dw, score, renorm, scale, bias=None):
    """Formula in 64 bits, by autograd on the definition."""
    x = torch.tensor(np.where(np.isneginf(logits), -1e300, logits), dtype=torch.float64, requires_grad=True)
    off = torch.tensor(np.isneginf(logits) if bias is None else (np.isneginf(logits) | np.isneginf(bias)[None]))
    xm = x.masked_fill(off, -1e300)
    s = torch.sigmoid(xm) if score == "sigmoid" else torch.softmax(xm, -1)
    live = torch.tensor(ids >= 0)
    c = s.gather(1, torch.tensor(ids).clamp(min=0)) * live
    if renorm:
        total = c.sum(-1, keepdim=True)
        c = c / torch.where(total > 0, total, 1.0)
    (c * scale * torch.tensor(dw, dtype=torch.float64)).sum().backward()
    return torch.nan_to_num(x.grad).masked_fill(off, 0.0).masked_fill(~live.any(-1, keepdim=True), 0.0).numpy()


def quantise(x):
    """x: float32 rows. The definition is in 32 bits, so this is too."""
    x = x.astype(np.float32)
    with np.errstate(all="ignore"):
        amax = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(x.shape[0], dtype=np.float32)
        bad = ~(amax < np.inf)
        use = ~bad & (amax >= np.float32(1e-30))
        inv = np.where(use, np.float32(1) / np.where(use, amax, np.float32(1)) * np.float32(127), np.float32(0)).astype(np.float32)
        q = np.rint(np.where(bad[:, None], np.float32(0), x) * inv[:, None])
        scale = np.where(bad, np.float32(np.nan), np.where(use, amax / np.float32(127), np.float32(0))).astype(np.float32)
    return q.astype(np.int8), scale


def matmul(a, sa, w, sw, bias=None, offsets=None):
    """y in 64 bits (sums in 64-bit integers), and the size of what is added, for tolerances. Rows outside all groups: NaN."""
    def dense(rows, scale, g):
        y = (rows.astype(np.int64) @ w[g].astype(np.int64).T).astype(np.float64) * scale[:, None].astype(np.float64) * sw[g][None].astype(np.float64)
        size = np.abs(y)
        if bias is not None:
            y, size = y + bias[g].astype(np.float64), size + np.abs(bias[g])
        return y, size
    if offsets is None:
        return dense(a, sa, 0)
    y = np.full((a.shape[0], w.shape[1]), np.nan)
    size = np.zeros_like(y)
    for g in range(w.shape[0]):
        lo, hi = int(offsets[g]), int(offsets[g + 1])
        if hi > lo:
            y[lo:hi], size[lo:hi] = dense(a[lo:hi], sa[lo:hi], g)
    return y, size
