"""GPU orthogonalised gradients on every form that a call can take (orth_cases: tiles of each shape, whole or in parts),
against the steps in 64 bits on the GPU.

Tolerance, by the norm of a matrix, as in test_gpu_orthogonalise.py: 8e-3 for five steps, 1e-3 for each step more; the
momentum is one fp32 multiply-add."""
import pytest

from tests import training_reference as R
from tests.orth_cases import CALLS

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2607_05116_amd import capi  # noqa: E402

COEF = [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]


def tol(steps):
    return 8e-3 + 1e-3 * max(0, steps - 5)


def steps64(u, steps=5, coef=None, eps=1e-7):
    x = u.double()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + eps)
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    for i in range(steps):
        a, b, c = R.QUINTIC if coef is None else coef[i]
        s = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * s + c * torch.bmm(s, s), x)
    return x.transpose(1, 2).contiguous() if tall else x


def run(g, steps=5, coef=None, eps=1e-7, momentum=None, mu=0.9, nesterov=True, shift=0):
    b, r, c = g.shape
    dt = capi.CAP_DTYPE_BF16 if g.dtype == torch.bfloat16 else capi.CAP_DTYPE_F32
    n = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=c, inter=r, max_rows=b)
    ws = torch.full((n,), 0x7E, dtype=torch.uint8, device="cuda")            # fp16 NaN everywhere
    out = torch.full((b * r * c + shift + 8,), 9.0, dtype=torch.bfloat16, device="cuda")
    got = out[shift:shift + b * r * c].view(b, r, c)
    if momentum is None:
        capi.cap_orthogonalise(dt, b, r, c, g, steps, coef, eps, got, ws)
    else:
        capi.cap_muon_update(dt, b, r, c, g, momentum, mu, nesterov, steps, coef, eps, got, ws)
    torch.cuda.synchronize()
    assert (out[:shift] == 9).all() and (out[shift + b * r * c:] == 9).all()  # nothing beside the result
    return got


def matrices(seed, b, r, c):
    gen = torch.Generator("cuda").manual_seed(seed)
    u = torch.randn((b, r, 8), generator=gen, device="cuda")
    v = torch.randn((b, 8, c), generator=gen, device="cuda")
    return 1e-3 * (torch.bmm(u, v) + torch.randn((b, r, c), generator=gen, device="cuda"))


def near(got, want, limit, names=None):
    err = ((got.double() - want).square().sum((1, 2)) / want.square().sum((1, 2))).sqrt()
    assert err.isfinite().all() and err.max().item() <= limit, err.max().item()


@pytest.mark.parametrize("b,r,c,steps", CALLS)
def test_forms(b, r, c, steps):
    g = matrices(b + r, b, r, c)
    near(run(g, steps), steps64(g, steps), tol(steps))


@pytest.mark.parametrize("b,r,c,steps", CALLS)
def test_forms_with_momentum(b, r, c, steps):
    g = matrices(b + c, b, r, c).bfloat16()
    m = 10 * matrices(b + c + 1, b, r, c)
    want = torch.tensor(0.9, dtype=torch.float32).double().item() * m.double() + g.double()
    got = run(g, steps, momentum=m)
    assert ((m.double() - want).abs().max() <= 2.0 ** -22 * want.abs().max()).item()
    near(got, steps64(g.double() + torch.tensor(0.9, dtype=torch.float32).double().item() * want, steps), tol(steps))


@pytest.mark.parametrize("b,r,c,steps", CALLS)
def test_low_ranks(b, r, c, steps):
    """One, two and a few directions among zeros, exactly; rows of very different size."""
    gen = torch.Generator("cuda").manual_seed(r)
    rank = torch.tensor([1, 2, 5], device="cuda").repeat(b)[:b]
    pick = (torch.arange(5, device="cuda")[None, :] < rank[:, None]).float()
    u = (torch.randn((b, r, 5), generator=gen, device="cuda") * pick[:, None, :]).bfloat16().float()
    u = u * torch.exp2(torch.randint(-3, 4, (b, r, 1), generator=gen, device="cuda").float())
    g = torch.bmm(u, torch.randn((b, 5, c), generator=gen, device="cuda").bfloat16().float())
    near(run(g, steps), steps64(g, steps), tol(steps) + 1.5 * 2.0 ** -23 * R.QUINTIC[0] ** steps)


@pytest.mark.parametrize("b,r,c,steps", [c for c in CALLS if c[0] > 1])
def test_a_matrix_of_zeros_and_one_with_nan_stay_alone(b, r, c, steps):
    """Whatever a tile reads of the next matrix past its own edge."""
    g = matrices(r, b, r, c)
    bad = min(1, b - 1)
    g[bad, r // 2, c // 3] = float("nan")
    zero = b - 1 if b > 2 else None
    if zero is not None:
        g[zero] = 0
    got = run(g, steps)
    assert got[bad].isnan().all() and (zero is None or not got[zero].any())
    keep = [i for i in range(b) if i not in (bad, zero)][:6]
    near(got[keep], steps64(g[keep], steps), tol(steps))
    g[bad, r // 2, c // 3] = float("inf")
    assert run(g, steps)[bad].isnan().all()


@pytest.mark.parametrize("b,r,c,steps", [(2, 200, 1000, 5), (3, 333, 517, 5), (2, 517, 333, 5), (32, 380, 383, 5), (48, 301, 381, 5),
                                         (3, 40, 701, 8), (48, 381, 251, 8)])
def test_shifted_tensors(b, r, c, steps):
    g = matrices(c, b, r, c)
    for dt in (torch.float32, torch.bfloat16):
        a = run(g.to(dt), steps)
        for shift in (1, 2, 4):
            buf = torch.zeros(g.numel() + shift, dtype=dt, device="cuda")
            buf[shift:] = g.to(dt).flatten()
            assert torch.equal(a, run(buf[shift:].view(b, r, c), steps, shift=shift)), shift
    m = matrices(c + 1, b, r, c)
    buf = torch.zeros(g.numel() + 1, device="cuda")
    buf[1:] = m.flatten()
    a = run(g, steps, momentum=m)
    assert torch.equal(a, run(g, steps, momentum=buf[1:].view(b, r, c))) and torch.equal(m.flatten(), buf[1:])


@pytest.mark.parametrize("b,r,c", [(2, 200, 1000), (3, 333, 517), (48, 500, 510), (32, 380, 384)])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
def test_step_counts(b, r, c, steps):
    g = matrices(steps, b, r, c)
    near(run(g, steps), steps64(g, steps), tol(steps))


@pytest.mark.parametrize("b,r,c", [(2, 200, 1000), (1, 6100, 1500), (48, 500, 510), (32, 380, 384)])
def test_own_coefficients(b, r, c):
    g = matrices(3, b, r, c)
    near(run(g, 3, COEF), steps64(g, 3, COEF), tol(3))


@pytest.mark.parametrize("b,r,c,steps", [(8, 2000, 2040, 5), (5, 1250, 5100, 5), (3, 1100, 1150, 5), (8, 1010, 1300, 7), (2, 200, 1000, 5)])
def test_same_bits_and_graph(b, r, c, steps):
    g = matrices(r, b, r, c)
    first = g.clone()
    a = run(g, steps)
    assert torch.equal(a, run(g, steps))
    out = torch.empty_like(a)
    n = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=c, inter=r, max_rows=b)
    ws = torch.full((n,), 0x7E, dtype=torch.uint8, device="cuda")
    call = lambda: capi.cap_orthogonalise(capi.CAP_DTYPE_F32, b, r, c, g, steps, None, 1e-7, out, ws)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        g.copy_(first.roll(i, 2))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
