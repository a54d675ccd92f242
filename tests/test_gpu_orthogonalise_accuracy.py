"""GPU orthogonalised gradients on matrices that are hard on their arithmetic: singular values of 0 (the gradient of
an expert with few tokens), energy in a few rows, against the steps in 64 bits.

Tolerance, by the norm of a matrix.  Where a singular value is 1 and others are 0, X <- p X + R X takes 3.4 X - 2.7 X:
R's rounding (2^-12 of an entry at most, a diagonal one none) and D's come out four times as large, on average over a
row's entries 5e-4 each; five steps with a slope of at most 1.2 leave 3.5e-3 at most, what X loses as an operand (2^-12
of an entry, times the share |p - a| of R in directions of 0, which each later step multiplies by a) 3e-3, the bf16
result 2^-9: 8e-3 in all.  (Where two or three entries are all there is, their roundings may agree: one such matrix in
1000 comes close to 1e-2.  The inputs here are fixed.)"""
import numpy as np
import pytest

from tests import training_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2607_05116_amd import capi  # noqa: E402

TOL = 8e-3


def matrix(kind, n, m, seed):
    """fp32 [n][m]; low ranks are exact (their factors are rounded, not the product)."""
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.standard_normal(s)                                     # noqa: E731
    bf = lambda a: torch.from_numpy(a).bfloat16().double().numpy()             # noqa: E731
    name, k = kind
    if name == "rank":
        g = bf(f(n, k)) @ bf(f(k, m))
    elif name == "uneven":
        g = bf(f(n, k) * np.exp(1.5 * f(n, 1))) @ bf(f(k, m))
    elif name == "rows":                     # k rows hold everything
        g = np.concatenate([f(k, m), np.zeros((n - k, m))])
    elif name == "outer":                    # k unequal rows, one direction
        g = np.concatenate([f(k, 1) @ f(1, m), np.zeros((n - k, m))])
    elif name == "plane":                    # k unequal rows, two directions
        g = np.concatenate([f(k, 2) @ f(2, m), np.zeros((n - k, m))])
    elif name == "beside":                   # one row over a floor
        g = np.concatenate([100 * f(1, m), 1e-3 * f(n - 1, m)])
    else:                                    # singular values that fall by e^-k
        u, v = np.linalg.qr(f(n, n))[0], np.linalg.qr(f(m, n))[0]
        g = (u * np.exp(-k * np.arange(n) / n)) @ v.T
    return (1e-3 * g).astype(np.float32)


KINDS = [("rank", 1), ("rank", 2), ("rank", 8), ("rank", 100), ("uneven", 1), ("uneven", 2), ("uneven", 8), ("rows", 1),
         ("rows", 3), ("outer", 2), ("outer", 4), ("plane", 3), ("plane", 4), ("beside", 1), ("fall", 12)]


def run(g, steps=5, coef=None, eps=1e-7):
    b, r, c = g.shape
    n = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=c, inter=r, max_rows=b)
    ws = torch.full((n,), 0x7E, dtype=torch.uint8, device="cuda")
    out = torch.empty((b, r, c), dtype=torch.bfloat16, device="cuda")
    capi.cap_orthogonalise(capi.CAP_DTYPE_F32, b, r, c, g, steps, coef, eps, out, ws)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def near(got, want, tol):
    for i in range(len(want)):
        err = np.linalg.norm(got[i] - want[i]) / np.linalg.norm(want[i])
        assert np.isfinite(got[i]).all() and err <= tol, f"matrix {i}: {err:.2e}"


@pytest.mark.parametrize("n,m", [(160, 160), (200, 1000), (256, 4096)])
@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}{k[1]}")
def test_hard_spectra(kind, n, m):
    host = np.stack([matrix((kind[0], min(kind[1], n)), n, m, s) for s in range(3)])
    near(run(torch.from_numpy(host).cuda()), [R.orth64(x) for x in host], TOL)
    tall = np.ascontiguousarray(host[:1].transpose(0, 2, 1))
    near(run(torch.from_numpy(tall).cuda()), [R.orth64(x) for x in tall], TOL)


@pytest.mark.parametrize("kind", [("rank", 1), ("rank", 300), ("uneven", 1), ("plane", 3)], ids=lambda k: f"{k[0]}{k[1]}")
def test_hard_spectra_of_many_tiles(kind):
    host = np.stack([matrix(kind, 1024, 1024, s) for s in range(2)])
    near(run(torch.from_numpy(np.concatenate([host] * 12)).cuda())[::13], [R.orth64(host[0]), R.orth64(host[1])], TOL)


@pytest.mark.parametrize("n,m", [(1, 50), (8, 30), (16, 64), (33, 100), (64, 64), (64, 200), (100, 300), (128, 128),
                                 (128, 1500)])
@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}{k[1]}")
def test_hard_spectra_of_few_rows(kind, n, m):
    host = np.stack([matrix((kind[0], min(kind[1], n)), n, m, s) for s in range(3)])
    near(run(torch.from_numpy(host).cuda()), [R.orth64(x) for x in host], TOL)
    tall = np.ascontiguousarray(host[:1].transpose(0, 2, 1))
    near(run(torch.from_numpy(tall).cuda()), [R.orth64(x) for x in tall], TOL)


@pytest.mark.parametrize("n,m", [(16, 40), (64, 100), (128, 300), (160, 200), (256, 1024)])
@pytest.mark.parametrize("size", [1.0, 1e-1, 1e-2, 1e-3, 1e-5, 1e-8, 1e-12])
def test_eps_above_the_norm(n, m, size):
    """|X0| = |U| / (|U| + eps) from 1 to 1e-12, for an ordinary matrix and one of rank 1."""
    for kind in (("rank", n), ("rank", 1)):
        host = matrix(kind, n, m, 5)[None]
        norm = float(np.linalg.norm(host.astype(np.float64)))
        eps = float(np.float32(norm * (1 / size - 1)))
        near(run(torch.from_numpy(host).cuda(), eps=eps), [R.orth64(host[0], eps=eps)], TOL)


def test_eps_of_each_matrix_of_a_batch():
    """Matrices of one call that eps leaves at their size, makes small and makes zeros of."""
    host = np.stack([matrix(("rank", 150), 150, 300, 6 + i) * np.float32(s) for i, s in enumerate((1e6, 1.0, 1e-6, 0.0))])
    for steps in (1, 2, 5):
        got = run(torch.from_numpy(host).cuda(), steps=steps, eps=1.0)
        near(got[:3], [R.orth64(x, steps, eps=1.0) for x in host[:3]], TOL)
        assert not got[3].any()


@pytest.mark.parametrize("n,m", [(1, 40), (16, 40), (64, 200), (128, 300), (200, 1000), (256, 1024)])
@pytest.mark.parametrize("steps", [6, 7, 8, 10])
def test_more_steps(n, m, steps):
    """1e-3 of arithmetic for each step more than five, and rounding to 22 bits (2^-23) that all steps multiply by a
    where a singular value is 0, of each step's X: 1.4 times the first one's."""
    tol = TOL + 1e-3 * (steps - 5) + 1.5 * 2.0 ** -23 * R.QUINTIC[0] ** steps
    for kind in KINDS:
        host = matrix((kind[0], min(kind[1], n)), n, m, 11)[None]
        near(run(torch.from_numpy(host).cuda(), steps), [R.orth64(host[0], steps)], tol)
    host = matrix(("rank", n), n, m, 12)[None]                                # tall
    tall = np.ascontiguousarray(host.transpose(0, 2, 1))
    near(run(torch.from_numpy(tall).cuda(), steps), [R.orth64(tall[0], steps)], tol)


def test_most_steps():
    """Sixteen: rounding rules where a singular value is 0, in any precision; others are as accurate as ever."""
    for n, m in ((100, 400), (200, 1000)):
        host = np.stack([matrix(("rank", n), n, m, s) for s in (1, 2)])
        near(run(torch.from_numpy(host).cuda(), 16), [R.orth64(x, 16) for x in host], TOL + 11e-3)
        low = matrix(("rank", 3), n, m, 3)[None]
        assert np.isfinite(run(torch.from_numpy(low).cuda(), 16)).all()


def test_steep_coefficients():
    """Four steps of the default and three that converge: a product of the a of 928; on both sides of 128 rows."""
    coef = [R.QUINTIC] * 4 + [(1.875, -1.25, 0.375)] * 3
    for n, m in ((64, 200), (128, 300), (200, 1000)):
        for kind in (("rank", n), ("rank", 1), ("uneven", 2), ("fall", 12)):
            host = matrix(kind, n, m, 4)[None]
            near(run(torch.from_numpy(host).cuda(), 7, coef), [R.orth64(host[0], 7, coef)], TOL)


@pytest.mark.parametrize("n,m", [(16, 40), (64, 100), (128, 300), (160, 200), (256, 1024)])
def test_range_of_the_norm(n, m):
    """|G| from 1e-15 to 1e18, eps = 0; beyond the range of fp32's squares NaN, and only in that matrix."""
    one = matrix(("rank", n), n, m, 7)
    one = (one / np.linalg.norm(one.astype(np.float64))).astype(np.float64)
    host = np.stack([one * s for s in (1e-15, 1e-9, 1.0, 1e9, 1e18)]).astype(np.float32)
    near(run(torch.from_numpy(host).cuda(), eps=0.0), [R.orth64(x, eps=0.0) for x in host], TOL)
    host = np.stack([one, one * 1e25, one]).astype(np.float32)
    got = run(torch.from_numpy(host).cuda())
    assert np.isnan(got[1]).all()
    near(got[::2], [R.orth64(host[0]), R.orth64(host[2])], TOL)


@pytest.mark.parametrize("n,m", [(160, 200), (300, 380), (131, 132)])
def test_an_odd_address_changes_no_bit(n, m):
    """Same inputs, same bits, also where the norm is summed without vector loads."""
    host = matrix(("rank", n), n, m, 8)[None]
    g = torch.from_numpy(host).cuda()
    a = run(g)
    for shift in (1, 2, 3):
        buf = torch.zeros(g.numel() + shift, device="cuda")
        buf[shift:] = g.flatten()
        assert np.array_equal(a, run(buf[shift:].view(1, n, m))), shift


@pytest.mark.parametrize("b,n,m", [(2500, 30, 60), (1025, 100, 128), (5, 20, 60000)])
def test_more_steps_of_large_batches(b, n, m):
    """Matrices that are taken in parts of the batch; the first, the last and some at every place between."""
    g = torch.randn((b, n, m), generator=torch.Generator("cuda").manual_seed(n), device="cuda")
    got = run(g, 6)
    some = sorted({0, 1, b // 3, b // 2, b - 2, b - 1})
    near(got[some], [R.orth64(x, 6) for x in g[some].cpu().numpy()], TOL + 1e-3)
    assert np.isfinite(got).all() and (np.abs(got).sum((1, 2)) > 0).all()
