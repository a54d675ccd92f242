"""GPU orthogonalised gradients (cap_orthogonalise, cap_muon_update) against the steps in 64 bits.

Tolerance, by the norm of a matrix: a step rounds S, b S + c S S and X as an operand to 11 bits, three relative errors
of at most 2^-12; the step's slope at singular values near 1 is at most 1.2, so five steps leave at most 4.4e-3, and
the bf16 result adds 2^-9: 6.4e-3, with the smaller singular values' share 8e-3.  The momentum is one fp32
multiply-add: 2^-23."""
import numpy as np
import pytest

from tests import training_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2607_05116_amd import capi  # noqa: E402

TOL = 8e-3


def _ws(batch, rows, cols):
    n = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=cols, inter=rows, max_rows=batch)
    return torch.full((n,), 0x7E, dtype=torch.uint8, device="cuda")          # fp16 NaN everywhere


def _run(g, steps=5, coef=None, eps=1e-7, momentum=None, mu=0.95, nesterov=True, stream=None, shift=0):
    b, r, c = g.shape
    dt = capi.CAP_DTYPE_BF16 if g.dtype == torch.bfloat16 else capi.CAP_DTYPE_F32
    out = torch.full((b * r * c + shift,), 9.0, dtype=torch.bfloat16, device="cuda")
    got = out[shift:].view(b, r, c)
    ws = _ws(b, r, c)
    torch.cuda.synchronize()
    if momentum is None:
        capi.cap_orthogonalise(dt, b, r, c, g, steps, coef, eps, got, ws, stream=stream)
    else:
        capi.cap_muon_update(dt, b, r, c, g, momentum, mu, nesterov, steps, coef, eps, got, ws, stream=stream)
    torch.cuda.synchronize()
    return got


def _matrix(seed, b, r, c, kind="plain"):
    rng = np.random.default_rng(seed)
    g = rng.standard_normal((b, r, c))
    if kind == "lowrank":
        q = min(4, r, c)
        g = g + 3 * rng.standard_normal((b, r, q)) @ rng.standard_normal((b, q, c))
    if kind == "rows":
        g = g * np.exp(1.5 * rng.standard_normal((b, r, 1)))
    if kind == "decay":
        u, _, v = np.linalg.svd(g, full_matrices=False)
        g = (u / np.arange(1, min(r, c) + 1)) @ v
    return (1e-3 * g).astype(np.float32)


def _near(got, want, tol=TOL):
    got = got.double().cpu().numpy()
    for i in range(len(want)):
        err, norm = np.linalg.norm(got[i] - want[i]), np.linalg.norm(want[i])
        assert np.isfinite(got[i]).all() and err <= tol * norm, f"matrix {i}: {err / norm:.2e}"


SHAPES = [(1, 1, 1), (2, 1, 7), (2, 7, 1), (1, 16, 16), (3, 17, 33), (2, 33, 17), (1, 64, 128), (1, 127, 129), (2, 129, 127),
          (1, 128, 2048), (5, 256, 128), (2, 200, 1000), (1, 333, 517), (1, 520, 300), (1, 768, 2048), (1, 1100, 640),
          (1, 16, 3000), (1, 2999, 3), (20, 65, 65), (1, 1025, 1030)]


@pytest.mark.parametrize("b,r,c", SHAPES)
@pytest.mark.parametrize("bf16", [False, True])
def test_orthogonalise(b, r, c, bf16):
    g = torch.from_numpy(_matrix(b + r + c, b, r, c))
    g = (g.bfloat16() if bf16 else g).cuda()
    host = g.double().cpu().numpy()
    _near(_run(g), [R.orth64(m) for m in host])


@pytest.mark.parametrize("kind", ["lowrank", "rows", "decay"])
@pytest.mark.parametrize("r,c", [(256, 256), (160, 640), (640, 160)])
def test_spectra(kind, r, c):
    host = _matrix(3, 2, r, c, kind)
    _near(_run(torch.from_numpy(host).cuda()), [R.orth64(m) for m in host])


@pytest.mark.parametrize("b,r,c", [(40, 640, 900), (40, 900, 640), (3, 1920, 2300), (24, 1024, 1024)])
def test_many_tiles(b, r, c):
    """Enough tiles for the large form of the products, with sides that end within a tile (reference: the same steps
    in 64 bits on the GPU)."""
    g = torch.randn((b, r, c), generator=torch.Generator("cuda").manual_seed(b + r), device="cuda")
    x = g.double()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    x = x.transpose(1, 2).contiguous() if r > c else x
    for _ in range(5):
        s = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = R.QUINTIC[0] * x + torch.matmul(R.QUINTIC[1] * s + R.QUINTIC[2] * torch.matmul(s, s), x)
    x = x.transpose(1, 2) if r > c else x
    err = ((_run(g).double() - x).square().sum((1, 2)) / x.square().sum((1, 2))).sqrt()
    assert err.max().item() <= TOL, err.max().item()


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("b,r,c", [(1, 5, 3), (3, 96, 200), (2, 300, 130), (1, 1024, 520)])
def test_muon_steps(b, r, c, nesterov):
    """Three updates in a row; the momentum is the state."""
    mom = torch.zeros((b, r, c), device="cuda")
    m = np.zeros((b, r, c))
    for i in range(3):
        g = torch.from_numpy(_matrix(10 + i, b, r, c)).bfloat16().cuda()
        host = g.double().cpu().numpy()
        got = _run(g, momentum=mom, mu=0.9, nesterov=nesterov)
        mu = float(np.float32(0.9))
        m = mu * m + host
        assert np.abs(mom.double().cpu().numpy() - m).max() <= 2.0 ** -22 * np.abs(m).max()
        u = host + mu * m if nesterov else m
        _near(got, [R.orth64(x) for x in u])


def test_coefficients_and_step_counts():
    host = _matrix(5, 2, 90, 140)
    g = torch.from_numpy(host).cuda()
    coef = [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]
    _near(_run(g, steps=3, coef=coef), [R.orth64(m, 3, coef) for m in host])
    for steps in (1, 2, 8):
        _near(_run(g, steps=steps), [R.orth64(m, steps) for m in host], TOL * max(1.0, steps / 5))


def test_eps_scale_and_range():
    """Gradients of any scale that fp32 squares hold; eps shows where it is as large as the norm."""
    for scale in (1e-12, 1.0, 1e12):
        host = (_matrix(6, 1, 48, 80) * scale).astype(np.float32)
        _near(_run(torch.from_numpy(host).cuda(), eps=0.0), [R.orth64(m, eps=0.0) for m in host])
    host = _matrix(6, 1, 48, 80)
    norm = float(np.linalg.norm(host[0]))
    _near(_run(torch.from_numpy(host).cuda(), eps=norm), [R.orth64(host[0], eps=norm)])


def test_a_matrix_of_zeros_and_one_with_nan_stay_alone():
    host = _matrix(7, 4, 70, 50)
    host[1] = 0.0
    host[2, 3, 4] = np.nan
    got = _run(torch.from_numpy(host).cuda()).float().cpu()
    assert not got[1].any() and got[2].isnan().all()
    for i in (0, 3):
        _near(got[i:i + 1], [R.orth64(host[i])])


@pytest.mark.parametrize("b,r,c", [(2, 33, 47), (2, 47, 33), (1, 128, 256)])
def test_unaligned_output(b, r, c):
    host = _matrix(8, b, r, c)
    g = torch.from_numpy(host).cuda()
    a = _run(g)
    for shift in (1, 2, 3):
        assert torch.equal(a, _run(g, shift=shift))


def test_unaligned_input():
    host = _matrix(9, 2, 31, 45)
    for dt in (torch.float32, torch.bfloat16):
        flat = torch.from_numpy(host).to(dt).cuda().flatten()
        buf = torch.cat([flat[:1], flat])
        assert torch.equal(_run(buf[1:].view(2, 31, 45)), _run(flat.view(2, 31, 45)))


def test_same_bits_streams_batch_and_graph():
    host = _matrix(10, 3, 256, 384)
    g = torch.from_numpy(host).cuda()
    a = _run(g)
    assert torch.equal(a, _run(g, stream=torch.cuda.Stream()))
    out, ws = torch.empty_like(a), _ws(3, 256, 384)
    mom = torch.zeros_like(g)

    def step():
        capi.cap_muon_update(capi.CAP_DTYPE_F32, 3, 256, 384, g, mom, 0.9, True, 5, None, 1e-7, out, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        g.copy_(torch.from_numpy(host).cuda() * (1 + i))
        mom.fill_(1e-3)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), mom.clone()
        mom.fill_(1e-3)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], mom)


def test_offsets_past_32_bits():
    """2.2e9 values: the last matrix, with zeros before it."""
    b, r, c = 33000, 256, 256
    g = torch.zeros((b, r, c), dtype=torch.bfloat16, device="cuda")
    last = torch.from_numpy(_matrix(11, 1, r, c)).bfloat16().cuda()
    g[-1] = last[0]
    out = torch.empty_like(g)
    n = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=c, inter=r, max_rows=b)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    capi.cap_orthogonalise(capi.CAP_DTYPE_BF16, b, r, c, g, 1, None, 1e-7, out, ws)
    torch.cuda.synchronize()
    _near(out[-1:], [R.orth64(last[0].double().cpu().numpy(), 1)])
    assert not out[-2].any().item() and not out[0].any().item()
