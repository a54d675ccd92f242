"""cap_route_scores where scores underflow, saturate or are equal, and where experts are off: the choice, the kept slots and
the gates of every token whose pruning the definition decides (scores_reference), which nearly all must be."""
import math

import numpy as np
import pytest

import scores_reference as ref
from test_gpu_route_scores import CASES, COST, PLAIN, SIGMOID, _grad, _route, capi  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

# relative: what two orders of fp64 operations on eight scores of a few ulp differ by is below 1e-14
NEAR = 1e-11
# scores from here on may be 0 or not
LEAST = 1e-299


def undecided(logits, idx, rank, R, node, p, kind, token_mask):
    """Per token: do two devices at or before the border of what is kept lie closer than NEAR, unless their slots have the
    same scores (then the lower device comes first), or does a sum come that close to 1 - p?"""
    T, k = idx.shape
    out = np.zeros(T, bool)
    target = 1.0 - float(np.float32(p))
    for t in range(T):
        on = np.isfinite(logits[t]) & (token_mask is None or bool(token_mask[t]))
        s = ref._scores(logits[t], on, kind)
        slots = {}
        for e in idx[t]:
            if on[e]:
                slots.setdefault(int(rank[e]), []).append(float(s[e]))
        values = [v for vs in slots.values() for v in vs]
        out[t] = any(0.0 < v < LEAST for v in values)
        if p == 0.0 or not slots:
            continue
        total = math.fsum(values)
        own = t // (T // R)
        share = {d: math.fsum(v) / total if total > 0.0 else 0.0 for d, v in slots.items()}
        far = {d: d // node != own // node for d in slots}
        worth = {d: math.inf if d == own else share[d] / (COST if far[d] else 1.0) for d in slots}
        order = sorted(slots, key=lambda d: (-worth[d], d))
        done = 0.0
        for a, b in zip(order, order[1:] + [None]):
            out[t] |= abs(done - target) < NEAR
            if done >= target:
                break
            done += share[a]
            if b is None or worth[a] == math.inf:
                continue
            alike = sorted(slots[a]) == sorted(slots[b]) and far[a] == far[b]
            out[t] |= worth[a] - worth[b] <= NEAR * worth[a] and worth[a] > 0.0 and not alike
    return out


def _all_decided(capi, logits, k, R, node, p, opt, bias=None, token_mask=None, rank=None):
    idx, w, keep, mask, rank = _route(capi, logits, k, R, node, p, opt, bias, token_mask, rank)
    r_idx, r_w, r_keep, r_mask, _ = ref.route(logits, k, rank, R, node, p, COST, bias=bias, token_mask=token_mask, **opt)
    assert np.array_equal(idx, r_idx)
    open_ = undecided(logits, r_idx, rank, R, node, p, opt["kind"], token_mask)
    assert open_.mean() <= 0.02
    sure = ~open_
    assert np.array_equal(keep[sure], r_keep[sure]) and np.array_equal(mask[sure], r_mask[sure])
    # one rounding to fp32, and the fp64 exponentials'; a softmax that is not normalised over the chosen is divided by a sum
    # of fp32 exponentials, which is within 2^-20
    rel = 2.0 ** -24 * (1 + 1e-6) + (2.0 ** -20 if opt["kind"] == "softmax" and not opt["normalise"] else 0.0)
    assert np.all(np.abs(w - r_w)[sure] <= rel * np.abs(r_w[sure]) + 2.0 ** -149)


BANDS = {"low": (-40, -20), "wide": (-300, 300), "lowest": (-3e38, -1e4), "alike": (-1e-30, 1e-30)}


@pytest.mark.parametrize("node", [8, 4])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.4])
@pytest.mark.parametrize("band", list(BANDS))
@pytest.mark.parametrize("opt", [dict(SIGMOID, n_groups=8, topk_groups=4, group_top=2), PLAIN, dict(kind="softmax", normalise=True)])
def test_extreme_logits(capi, opt, band, p, node):  # noqa: F811
    rng = np.random.default_rng(5)
    logits = rng.uniform(*BANDS[band], (64, 64)).astype(np.float32)
    if opt["kind"] == "sigmoid":
        logits = np.minimum(logits, 30)            # above, different logits have one score in 64 bits
        if band == "lowest":
            logits = rng.uniform(-690, -600, (64, 64)).astype(np.float32)
    _all_decided(capi, logits, 8, 8, node, p, opt)


@pytest.mark.parametrize("p", [0.0, None])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_experts_off_and_tokens_masked(capi, case, p):  # noqa: F811
    E, k, R, each, node, p_case, opt, biased = CASES[case]
    rng = np.random.default_rng(300 + case)
    T = R * each
    logits = (2.0 * rng.standard_normal((T, E))).astype(np.float32)
    logits[rng.random((T, E)) < 0.5] = -math.inf
    logits[rng.random((T, E)) < 0.05] = math.nan
    logits[rng.random((T, E)) < 0.02] = math.inf
    logits[rng.random(T) < 0.2] = -math.inf
    token_mask = (rng.random(T) < 0.8).astype(np.uint8)
    logits[token_mask == 0] = rng.choice(np.array([math.nan, math.inf, -math.inf, 3e38], np.float32), (int((token_mask == 0).sum()), E))
    bias = (0.3 * rng.standard_normal(E)).astype(np.float32) if biased else None
    rank = rng.permutation(np.arange(E, dtype=np.int32) // (E // R)).astype(np.int32)
    _all_decided(capi, logits, k, R, node, p_case if p is None else p, opt, bias, token_mask, rank)


# ------------------------------------------------------------------ the gradient at any scale
@pytest.mark.parametrize("scale", [1e-44, 1e-39, 2.0 ** -128, 2.0 ** -126, 1e-30, 2.5, 1e30, 2.0 ** 127, 3.4e38])
@pytest.mark.parametrize("kind,normalise", [("sigmoid", True), ("sigmoid", False), ("softmax", True), ("softmax", False)])
def test_gradient_at_the_ends_of_the_scales(capi, kind, normalise, scale):  # noqa: F811
    """Finite scales above 0, whose inverse need not be a number of fp32."""
    T, E, k = 40, 32, 4
    rng = np.random.default_rng(11)
    logits = (2.0 * rng.standard_normal((T, E))).astype(np.float32)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    keep = (rng.random((T, k)) < 0.8).astype(np.uint8)
    d_w = (rng.standard_normal((T, k)) / 64).astype(np.float32)
    scale = float(np.float32(scale))
    opt = dict(kind=kind, normalise=normalise, scale=scale)
    w64 = ref.gates(logits.astype(np.float64), idx, keep, kind, normalise, scale)
    got = _grad(capi, logits, idx, keep, w64.astype(np.float32), d_w, opt, None, False).astype(np.float64)
    want = ref.grad(logits.astype(np.float64), idx, keep, d_w.astype(np.float64), kind, normalise, scale)
    assert np.isfinite(got).all()
    # what test_grad counts, and what is lost below the least normal number: a gate is off by 2^-150 there, and so is each
    # product; the gates over the scale are at most 1 + 2^-150 / scale, the sum of four products over it that of |d_w|
    terms = np.abs(w64 * d_w * keep)
    least = 2.0 ** -149
    share = np.abs(w64) / scale + least / scale
    size, lost = np.zeros((T, E)), np.zeros((T, E))
    np.put_along_axis(size, idx, terms + share * terms.sum(1, keepdims=True), 1)
    rounding = least * (2.0 + np.abs(d_w))                       # of w d_w
    np.put_along_axis(lost, idx, rounding + share * rounding.sum(1, keepdims=True) + least * (np.abs(d_w).sum(1, keepdims=True) + 2.0), 1)
    if kind == "softmax" and not normalise:
        size += terms.sum(1, keepdims=True)
        lost += rounding.sum(1, keepdims=True) + 2 * least
    assert np.all(np.abs(got - want) <= 32 * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(want) + 4 * lost + 2.0 ** -49 * terms.sum(1, keepdims=True))
