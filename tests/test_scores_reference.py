"""The 64-bit reference of routing by scores: its gradient against differences, its e4m3 against torch's type."""
import numpy as np
import pytest
import torch

import scores_reference as ref


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("normalise", [True, False])
def test_gradient_against_differences(kind, normalise):
    rng = np.random.default_rng(1)
    T, E, k, h = 4, 12, 5, 1e-6
    x = rng.standard_normal((T, E))
    x[1, :3] = -np.inf
    idx = np.stack([3 + rng.permutation(E - 3)[:k] for _ in range(T)])
    keep = (rng.random((T, k)) < 0.7).astype(np.uint8)
    d_w = rng.standard_normal((T, k))
    got = ref.grad(x, idx, keep, d_w, kind, normalise, 2.5)
    for e in range(E):
        step = np.zeros(E)
        step[e] = h
        up, down = (ref.gates(x + s * step, idx, keep, kind, normalise, 2.5) for s in (1, -1))
        # the third derivative's h^2 and rounding over h: below 1e-9 and 1e-9
        assert np.allclose(((up - down) * d_w).sum(1) / (2 * h), got[:, e], atol=1e-8)


def test_rounding_is_torch_e4m3():
    rng = np.random.default_rng(2)
    codes = ref.code_values()
    assert np.array_equal(torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy(), codes.astype(np.float32), equal_nan=True)
    v = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 0.02]).astype(np.float32)
    half = np.sort(codes[np.isfinite(codes)])
    v = np.concatenate([v, ((half[1:] + half[:-1]) / 2).astype(np.float32)])
    assert np.array_equal(torch.from_numpy(v).to(torch.float8_e4m3fn).float().numpy(), ref.round_e4m3(v).astype(np.float32))


def test_scales():
    for top, want in [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 2.0 ** -126), (2.0 ** -140, 2.0 ** -126),
                      (1.75, 2.0 ** -8), (1.7500001, 2.0 ** -7), (3.4e38, 2.0 ** 120)]:
        assert ref.block_scale(top) == want, top
