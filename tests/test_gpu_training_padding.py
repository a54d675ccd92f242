"""Padding tokens of a router's training step, whatever their rows of x hold (paper_2607_05116_amd.training)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from tests.test_gpu_training import K, T, _batch, _trainer  # noqa: E402

CASES = {"mask": ([0, 100, 100, 700, T], 5), "offsets": ([37, 100, 100, 700, 911], 0), "both": ([37, 100, 100, 700, 911], 5)}


def _left_out(offsets, every):
    t = torch.arange(T, device="cuda")
    out = (t < offsets[0]) | (t >= offsets[-1])
    mask = None
    if every:
        mask = (t % every != 0).to(torch.uint8)
        out = out | (mask == 0)
    return out, mask


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_rows_that_count_nowhere(case, apart, value):
    """The weights after two steps are those of zeros in these rows, bit for bit, and x stays as it is."""
    offsets, every = CASES[case]
    out, mask = _left_out(offsets, every)
    offs = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    d_gates = torch.randn((T, K), generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    a, b = _trainer(), _trainer()
    for i in range(2):
        x = _batch(20 + i)
        clean, dirty = x.clone(), x.clone()
        clean[out] = 0
        dirty[out] = value
        before = dirty.clone()
        a.step(clean, d_gates, offs, mask)
        if apart:
            b.forward(dirty, offs, mask)
            b.backward(dirty, d_gates, offs, mask)
            b.opt.step(b.w, b.d_w, b.w_bf16)
        else:
            b.step(dirty, d_gates, offs, mask)
        torch.cuda.synchronize()
        assert torch.equal(dirty.view(torch.int16), before.view(torch.int16))
    for n in ("loss", "counts", "d_w", "w", "w_bf16"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n
    assert a.w.isfinite().all()
