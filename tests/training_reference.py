"""The training operators in 64 bits, from their definitions (numpy)."""
import numpy as np

QUINTIC = (3.4445, -4.7750, 2.0315)


def softmax64(logits, mask=None, offsets=None):
    """P, lse, valid and the sequence (-1: none) of every token; rows of tokens that are not valid are 0."""
    x = np.asarray(logits, np.float64)
    T = x.shape[0]
    offs = np.array([0, T]) if offsets is None else np.asarray(offsets, np.int64)
    S = len(offs) - 1
    seq = np.searchsorted(offs, np.arange(T), side="right") - 1
    seq[seq >= S] = -1
    valid = seq >= 0
    if mask is not None:
        valid = valid & (np.asarray(mask) != 0)
    valid = valid & (np.nan_to_num(x, nan=-np.inf, posinf=np.inf, neginf=-np.inf).max(1, initial=-np.inf) > -np.inf)
    P, lse = np.zeros_like(x), np.zeros(T)
    for t in np.nonzero(valid)[0]:
        top = x[t].max()
        e = np.exp(x[t] - top)
        P[t], lse[t] = e / e.sum(), top + np.log(e.sum())
    return P, lse, valid, seq, S


def balance64(logits, idx, keep=None, mask=None, offsets=None, balance_coef=1.0, z_coef=1.0):
    T, k = idx.shape
    E = logits.shape[1]
    P, lse, valid, seq, S = softmax64(logits, mask, offsets)
    counts, probs, n = np.zeros((S, E), np.int64), np.zeros((S, E)), np.zeros(S, np.int64)
    for t in np.nonzero(valid)[0]:
        s = seq[t]
        n[s] += 1
        probs[s] += P[t]
        for j in range(k):
            if (keep is None or keep[t, j]) and 0 <= idx[t, j] < E:
                counts[s, idx[t, j]] += 1
    m = np.maximum(n, 1)[:, None]
    probs /= m
    present, total = int((n > 0).sum()), int(n.sum())
    balance = (E / (k * m) * counts * probs).sum() / max(present, 1)
    z = (lse[valid] ** 2).sum() / max(total, 1)
    tokens = np.concatenate([n, [present, total]])
    return dict(counts=counts, probs=probs, tokens=tokens,
                loss=np.array([balance_coef * balance + z_coef * z, balance, z]))


def grad64(logits, idx, keep, w, d_w, mask=None, offsets=None, balance_coef=1.0, z_coef=1.0, d_loss=1.0):
    T, k = idx.shape
    E = logits.shape[1]
    P, lse, valid, seq, S = softmax64(logits, mask, offsets)
    f = balance64(logits, idx, keep, mask, offsets)
    n, present, total = f["tokens"][:S], f["tokens"][S], f["tokens"][S + 1]
    out = np.zeros((T, E))
    for t in np.nonzero(valid)[0]:
        s = seq[t]
        C = balance_coef * E * f["counts"][s] / (k * float(n[s]) ** 2 * present)
        out[t] = d_loss * (P[t] * (C - (P[t] * C).sum()) + 2 * z_coef * lse[t] / total * P[t])
        if d_w is not None:
            kept = np.ones(k, bool) if keep is None else keep[t] != 0
            ww, dd = w[t].astype(np.float64) * kept, np.where(kept, d_w[t], 0).astype(np.float64)
            np.add.at(out[t], idx[t][kept], (ww * (dd - (ww * dd).sum()))[kept])
    return out


def orth64(u, steps=5, coef=None, eps=1e-7):
    x = np.asarray(u, np.float64)
    x = x / (np.linalg.norm(x) + eps)
    for i in range(steps):
        a, b, c = QUINTIC if coef is None else coef[i]
        g = x @ x.T if x.shape[0] <= x.shape[1] else x.T @ x
        p = b * g + c * (g @ g)
        x = a * x + (p @ x if x.shape[0] <= x.shape[1] else x @ p)
    return x
