"""Routing by scores and its gradient in 64 bits, token by token from the definition (numpy; no code of the package),
and e4m3 rounding with its block scales."""
import math

import numpy as np

CLOSE = 1e-11        # closer decisions than this are the rounding's


def _scores(row, on, kind):
    """Scores of the experts that are on, 0 for others."""
    s = np.zeros(len(row))
    if not on.any():
        return s
    x = row[on].astype(np.float64)
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            s[on] = 1.0 / (1.0 + np.exp(-x))
    else:
        e = np.exp(x - x.max())
        s[on] = e / e.sum()
    return s


def route(logits, k, expert_rank, R, node, p, cost, kind="softmax", n_groups=1, topk_groups=1, group_top=1, normalise=True,
          scale=1.0, bias=None, token_mask=None):
    """idx, w (fp64), keep, mask, and per token whether pruning came down to values closer than CLOSE."""
    T, E = logits.shape
    size = E // n_groups
    idx, w = np.zeros((T, k), np.int32), np.zeros((T, k))
    keep, mask, close = np.zeros((T, k), np.uint8), np.zeros(T, np.uint64), np.zeros(T, bool)
    target = 1.0 - float(np.float32(p))
    for t in range(T):
        row = logits[t]
        on = np.isfinite(row)
        if token_mask is not None and not token_mask[t]:
            on = np.zeros(E, bool)
        s = _scores(row, on, kind)
        biased = s + (bias.astype(np.float64) if bias is not None else 0.0)
        key = biased if bias is not None else np.where(on, row, 0.0).astype(np.float64)
        open_ = np.ones(E, bool)
        if topk_groups < n_groups:
            totals = []
            for g in range(n_groups):
                member = [e for e in range(g * size, (g + 1) * size) if on[e]]
                # single experts without a bias go by their logits
                value = row.astype(np.float64) if bias is None and (group_top == 1 or size == 1) else biased
                best = sorted((value[e] for e in member), reverse=True)[:group_top]
                totals.append(sum(best) if best else -math.inf)
            chosen = sorted(range(n_groups), key=lambda g: (-totals[g], g))[:topk_groups]
            open_ = np.isin(np.arange(E) // size, chosen)
        order = sorted(range(E), key=lambda e: (not open_[e], not on[e], -key[e] if on[e] else 0.0, e))[:k]
        idx[t] = order
        live = [s_ for s_ in range(k) if on[order[s_]]]
        q = np.array([s[e] for e in order])
        total = sum(q[s_] for s_ in live)
        share = [q[s_] / total if total > 0 else 0.0 for s_ in range(k)]
        devices = {}
        for s_ in live:
            d = int(expert_rank[order[s_]])
            devices[d] = devices.get(d, 0.0) + share[s_]
        kept = set(devices)
        if p > 0:
            own = t // (T // R)
            worth = {d: math.inf if d == own else a / (cost if d // node != own // node else 1.0)
                     for d, a in devices.items()}
            ranked = sorted(devices, key=lambda d: (-worth[d], d))
            finite = [worth[d] for d in ranked if worth[d] < math.inf]
            close[t] = any(a - b < CLOSE for a, b in zip(finite, finite[1:]))
            cum, kept = 0.0, set()
            for d in ranked:
                close[t] |= abs(cum - target) < CLOSE
                if cum >= target:
                    break
                kept.add(d)
                cum += devices[d]
        for s_ in live:
            if int(expert_rank[order[s_]]) in kept:
                keep[t, s_] = 1
        for d in kept:
            mask[t] |= np.uint64(1 << d)
        sum_kept = sum(q[s_] for s_ in range(k) if keep[t, s_])
        for s_ in range(k):
            if keep[t, s_]:
                w[t, s_] = scale * q[s_] / (sum_kept if normalise else 1.0) if sum_kept > 0 or not normalise else 0.0
    return idx, w, keep, mask, close


def gates(x, idx, keep, kind, normalise, scale):
    """Gates of given choices from fp64 logits."""
    T, k = idx.shape
    w = np.zeros((T, k))
    for t in range(T):
        s = _scores(x[t], np.isfinite(x[t]), kind)
        q = np.where(keep[t] != 0, s[idx[t]], 0.0)
        total = q.sum() if normalise else 1.0
        w[t] = scale * q / total if total > 0 else 0.0
    return w


def grad(x, idx, keep, d_w, kind, normalise, scale):
    """Gradient of sum(w d_w) with respect to the logits, from the quotient rule on scores."""
    T, E = x.shape
    out = np.zeros((T, E))
    for t in range(T):
        on = np.isfinite(x[t])
        s = _scores(x[t], on, kind)
        kept = [j for j in range(idx.shape[1]) if keep[t, j]]
        ds = np.zeros(E)                           # gradient at the scores
        total = sum(s[idx[t, j]] for j in kept)
        if not kept or (normalise and total <= 0):
            continue
        for j in kept:
            if normalise:
                mean = sum(s[idx[t, i]] / total * d_w[t, i] for i in kept)
                ds[idx[t, j]] = scale / total * (d_w[t, j] - mean)
            else:
                ds[idx[t, j]] = scale * d_w[t, j]
        out[t] = ds * s * (1.0 - s) if kind == "sigmoid" else s * (ds - (s * ds).sum())
    return out


# ------------------------------------------------------------------ e4m3
def code_values():
    """The value of each of the 256 codes."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v[c] = math.ldexp(1.0 + m / 8.0, e - 7) if e else math.ldexp(m / 8.0, -6)
        if (c & 0x7F) == 0x7F:
            v[c] = math.nan
        elif c & 0x80:
            v[c] = -v[c]
    return v


def round_e4m3(v):
    """Nearest e4m3 value, ties to the even mantissa, for |v| <= 448."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(np.abs(v))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(v / step) * step


def block_scale(top):
    """The least power of two, from 2^-126 on, with which `top` is at most 448."""
    m, e = np.frexp(np.asarray(top, np.float64))          # top = m 2^e, 1/2 <= m < 1;  448 = 7/8 2^9
    e = np.where(top == 0, -2000, np.where(m <= 0.875, e - 9, e - 8))
    return np.ldexp(1.0, np.maximum(e, -126))


def quantise(x, block_rows):
    """Rounded quotients and scales of a matrix [rows][cols]; what is not finite becomes NaN and sets no scale."""
    rows, cols = x.shape
    nb = -(-rows // block_rows)
    q, scale = np.zeros((rows, cols)), np.zeros((nb, cols // 128))
    x = x.astype(np.float64)
    for b in range(nb):
        for c in range(cols // 128):
            part = x[b * block_rows:(b + 1) * block_rows, c * 128:(c + 1) * 128]
            finite = np.isfinite(part)
            scale[b, c] = block_scale(np.abs(part[finite]).max() if finite.any() else 0.0)
            with np.errstate(invalid="ignore"):
                r = round_e4m3(np.where(finite, part, 0.0) / scale[b, c])
            q[b * block_rows:(b + 1) * block_rows, c * 128:(c + 1) * 128] = np.where(finite, r, math.nan)
    return q, scale
