"""GPU load-balance loss and router gradient (cap_balance_loss, cap_router_grad) against their definitions in 64 bits.

Tolerances.  A probability has the error of its exponential (argument up to 30, rounded at 2^-24, and two units of the
hardware's exponential) and of a sum of at most 256 terms: below 5e-6 of its value; sums over tokens add less than
that.  Compared by norm, 1e-5.  bf16 outputs add half a unit in the last place, 2^-9 of each value."""
import numpy as np
import pytest

from tests import training_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2607_05116_amd import capi  # noqa: E402

TOL = 1e-5


def _case(seed, T, E, k, offsets=None, masked=False, pruned=True, scale=1.5):
    rng = np.random.default_rng(seed)
    logits = (scale * rng.standard_normal((T, E))).astype(np.float32)
    idx = np.argsort(-logits, 1, kind="stable")[:, :k].astype(np.int32)
    top = np.take_along_axis(logits, idx, 1).astype(np.float64)
    keep = (rng.random((T, k)) < 0.7).astype(np.uint8) if pruned else np.ones((T, k), np.uint8)
    keep[:, 0] = 1
    w = np.exp(top - top[:, :1]) * keep
    w = (w / w.sum(1, keepdims=True)).astype(np.float32)
    d_w = rng.standard_normal((T, k)).astype(np.float32)
    mask = (rng.random(T) < 0.8).astype(np.uint8) if masked else None
    return dict(logits=logits, idx=idx, keep=keep, w=w, d_w=d_w, mask=mask, offsets=offsets)


def _dev(a, shift=0):
    """On the GPU; shift > 0: that many elements past an aligned start."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a))
    if not shift:
        return t.cuda()
    buf = torch.zeros(t.numel() + shift, dtype=t.dtype, device="cuda")
    buf[shift:] = t.flatten().cuda()
    return buf[shift:].view(t.shape)


def _forward(c, bc=0.7, zc=0.3, shift=0, stream=None, keep=True):
    T, k = c["idx"].shape
    E = c["logits"].shape[1]
    S = 1 if c["offsets"] is None else len(c["offsets"]) - 1
    d = {n: _dev(c[n], shift) for n in ("logits",)}
    d.update({n: _dev(c[n]) for n in ("idx", "keep", "w", "d_w", "mask")})
    d["offs"] = None if c["offsets"] is None else _dev(np.asarray(c["offsets"], np.int32))
    o = dict(counts=torch.full((S, E), -7, dtype=torch.int32, device="cuda"), probs=torch.full((S, E), 9.0, device="cuda"),
             tokens=torch.full((S + 2,), -7, dtype=torch.int32, device="cuda"), loss=torch.full((3,), 9.0, device="cuda"))
    n = capi.cap_workspace_size(capi.CAP_OP_BALANCE_LOSS, capi.Topology(E=E, T=T), max_rows=S)
    ws = torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")            # contents need no initialisation
    torch.cuda.synchronize()
    capi.cap_balance_loss(T, k, E, d["logits"], d["idx"], d["keep"] if keep else None, d["mask"], d["offs"], S, bc, zc,
                          o["counts"], o["probs"], o["tokens"], o["loss"], ws, stream=stream)
    torch.cuda.synchronize()
    return d, o, S


def _backward(c, d, o, S, bc=0.7, zc=0.3, bf16=False, up=None, shift=0, gates=True, keep=True):
    T, k = c["idx"].shape
    E = c["logits"].shape[1]
    out = torch.full((T * E + shift,), 9.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")[shift:].view(T, E)
    capi.cap_router_grad(T, k, E, d["logits"], d["idx"], d["keep"] if keep else None, d["w"], d["d_w"] if gates else None,
                         d["mask"], d["offs"], S, o["counts"], o["tokens"], bc, zc, up,
                         capi.CAP_DTYPE_BF16 if bf16 else capi.CAP_DTYPE_F32, out)
    torch.cuda.synchronize()
    return out


def _near(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    err, norm = np.linalg.norm(got - want), np.linalg.norm(want)
    assert np.isfinite(got).all(), what
    assert err <= tol * norm + 1e-30, f"{what}: {err / max(norm, 1e-300):.2e}"


def _check_forward(c, o, bc=0.7, zc=0.3):
    ref = R.balance64(c["logits"], c["idx"], c["keep"], c["mask"], c["offsets"], bc, zc)
    assert np.array_equal(o["counts"].cpu().numpy(), ref["counts"])
    assert np.array_equal(o["tokens"].cpu().numpy(), ref["tokens"])
    _near(o["probs"].cpu().numpy(), ref["probs"], TOL, "probs")
    _near(o["loss"].cpu().numpy(), ref["loss"], TOL, "loss")


def _ragged(T, S, seed):
    cuts = np.sort(np.random.default_rng(seed).integers(0, T + 1, S - 1))
    return [0, *cuts.tolist(), T]


SHAPES = [  # T, E, k, offsets, masked
    (1, 1, 1, None, False), (1, 16, 2, [0, 1], False), (2, 5, 3, [0, 1, 2], False), (3, 256, 8, None, True),
    (63, 17, 2, None, False), (64, 64, 6, [0, 64], False), (65, 65, 4, [0, 64, 65], True), (130, 128, 8, None, True),
    (257, 129, 8, [0, 0, 16, 16, 17, 80, 250, 257, 257], True), (300, 250, 7, _ragged(300, 40, 1), False),
    (1000, 256, 8, _ragged(1000, 300, 2), True), (4097, 64, 6, _ragged(4097, 9, 3), False),
    (5000, 40, 8, _ragged(5000, 2000, 4), True), (16384, 16, 2, [0, 16384], False),
    (16500, 33, 3, _ragged(16500, 12, 5), True), (20000, 128, 8, [0, 64, 128, 129, 12800, 12928, 20000], False)]


@pytest.mark.parametrize("T,E,k,offsets,masked", SHAPES)
def test_loss_and_gradient(T, E, k, offsets, masked):
    c = _case(T + E, T, E, k, offsets, masked)
    d, o, S = _forward(c)
    _check_forward(c, o)
    want = R.grad64(c["logits"], c["idx"], c["keep"], c["w"], c["d_w"], c["mask"], c["offsets"], 0.7, 0.3)
    _near(_backward(c, d, o, S).cpu().numpy(), want, TOL, "d_logits")
    got = _backward(c, d, o, S, bf16=True).float().cpu().numpy()
    assert np.all(np.abs(got - want) <= np.abs(want) * 2.0 ** -8 + TOL * np.abs(want).max())
    # the balance part alone, scaled by the gradient that arrives at the loss
    up = torch.tensor(-2.5, device="cuda")
    want = R.grad64(c["logits"], c["idx"], c["keep"], None, None, c["mask"], c["offsets"], 0.7, 0.3, -2.5)
    _near(_backward(c, d, o, S, up=up, gates=False).cpu().numpy(), want, TOL, "d_logits of the loss")


@pytest.mark.parametrize("E", [64, 96, 250])
def test_unaligned_buffers(E):
    c = _case(5, 200, E, 4, _ragged(200, 5, 6), True)
    d, o, S = _forward(c, shift=1)
    _check_forward(c, o)
    want = R.grad64(c["logits"], c["idx"], c["keep"], c["w"], c["d_w"], c["mask"], c["offsets"], 0.7, 0.3)
    for bf16 in (False, True):
        got = _backward(c, d, o, S, bf16=bf16, shift=1).float().cpu().numpy()
        assert np.all(np.abs(got - want) <= np.abs(want) * (2.0 ** -8 if bf16 else 0) + TOL * np.abs(want).max())


def test_no_keep_array_keeps_every_slot():
    c = _case(7, 333, 48, 5, None, False, pruned=False)
    d, o, S = _forward(c, keep=False)
    _check_forward(c, o)
    want = R.grad64(c["logits"], c["idx"], None, c["w"], c["d_w"], None, None, 0.7, 0.3)
    _near(_backward(c, d, o, S, keep=False).cpu().numpy(), want, TOL, "d_logits")


def test_masked_rows_hold_anything():
    """NaN, infinities and experts out of range in padding tokens; -inf and the lowest value in valid ones."""
    c = _case(8, 400, 70, 4, _ragged(400, 6, 7), True)
    x, mask = c["logits"], c["mask"]
    pad = np.nonzero(mask == 0)[0]
    x[pad[0::4]], x[pad[1::4]], x[pad[2::4]] = np.nan, np.inf, -np.inf
    c["idx"][pad[3::4]] = 10 ** 6
    live = np.nonzero(mask)[0]
    x[live[0], 5:] = -np.inf                       # few experts switched on
    x[live[1], 1:] = -np.inf                       # one
    x[live[2]] = -np.inf                           # none: the token is not valid
    x[live[3]] = np.finfo(np.float32).min          # all at the lowest value: uniform
    x[live[4], ::2] = np.finfo(np.float32).min
    c["idx"][live[5], 1] = 70                      # out of range: ignored
    c["idx"][live[6], 2] = -1
    c["keep"][live[5], 1] = c["keep"][live[6], 2] = 0
    d, o, S = _forward(c, zc=0.0)
    x = np.where(mask[:, None] != 0, x, 0.0)       # the reference's masked rows are ordinary
    ref = R.balance64(x, c["idx"], c["keep"], mask, c["offsets"], 0.7, 0.0)
    assert np.array_equal(o["counts"].cpu().numpy(), ref["counts"])
    assert np.array_equal(o["tokens"].cpu().numpy(), ref["tokens"])
    _near(o["probs"].cpu().numpy(), ref["probs"], TOL, "probs")
    _near(o["loss"].cpu().numpy()[:2], ref["loss"][:2], TOL, "loss")
    got = _backward(c, d, o, S, zc=0.0).cpu().numpy()
    want = R.grad64(x, np.clip(c["idx"], 0, 69), c["keep"], c["w"], c["d_w"], mask, c["offsets"], 0.7, 0.0)
    _near(got, want, TOL, "d_logits")
    assert not got[pad].any() and not got[live[2]].any()


def test_tokens_outside_the_sequences_count_nowhere():
    c = _case(9, 500, 32, 4, [37, 100, 100, 411], False)
    d, o, S = _forward(c)
    _check_forward(c, o)
    got = _backward(c, d, o, S).cpu().numpy()
    want = R.grad64(c["logits"], c["idx"], c["keep"], c["w"], c["d_w"], None, c["offsets"], 0.7, 0.3)
    _near(got, want, TOL, "d_logits")
    assert not got[:37].any() and not got[411:].any()


@pytest.mark.parametrize("T,offsets", [(0, None), (0, [0, 0, 0]), (40, [0, 40])])
def test_no_valid_token(T, offsets):
    c = _case(10, max(T, 1), 24, 3, offsets, False)
    c = {n: (v[:T] if isinstance(v, np.ndarray) else v) for n, v in c.items()}
    c["mask"] = np.zeros(T, np.uint8)
    d, o, S = _forward(c)
    assert not any(o[n].any().item() for n in o)
    if T:
        assert not _backward(c, d, o, S).any().item()


def test_gradient_against_differences():
    """Along its own direction, through the kernel's own loss (fp32: its rounding over the step, 1e-7 / 0.04 of
    values near 1, and the step's square are below 2e-3 of the slope)."""
    c = _case(11, 24, 16, 3, [0, 10, 24], False)
    d, o, S = _forward(c)
    g = _backward(c, d, o, S, gates=False).double().cpu().numpy()
    n = np.linalg.norm(g)
    loss = lambda h: _forward(dict(c, logits=(c["logits"] + h * g / n).astype(np.float32)))[1]["loss"][0].item()  # noqa: E731
    slope = (loss(0.02) - loss(-0.02)) / 0.04
    assert abs(slope - n) <= 5e-3 * n, (slope, n)


def test_gates_gradient_against_differences():
    """The gates' part, against differences of the kept softmax in 64 bits."""
    c = _case(12, 30, 20, 5, None, False)
    d, o, S = _forward(c, 0.0, 0.0)
    got = _backward(c, d, o, S, 0.0, 0.0).double().cpu().numpy()

    def value(x):
        top = np.take_along_axis(x, c["idx"].astype(np.int64), 1)
        e = np.exp(top - top.max(1, keepdims=True)) * c["keep"]
        return (e / e.sum(1, keepdims=True) * c["d_w"]).sum()

    x = c["logits"].astype(np.float64)
    rng = np.random.default_rng(1)
    for t, e in zip(rng.integers(0, 30, 60), rng.integers(0, 20, 60)):
        h = np.zeros_like(x)
        h[t, e] = 1e-5
        assert abs((value(x + h) - value(x - h)) / 2e-5 - got[t, e]) <= 1e-5


def test_same_bits_streams_and_graph():
    c = _case(13, 6000, 96, 6, _ragged(6000, 50, 8), True)
    _, a, _ = _forward(c)
    side = torch.cuda.Stream()
    d, b, S = _forward(c, stream=side)
    for n in a:
        assert torch.equal(a[n], b[n]), n
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    out = torch.empty((6000, 96), device="cuda")

    def both():
        capi.cap_balance_loss(6000, 6, 96, d["logits"], d["idx"], d["keep"], d["mask"], d["offs"], S, 0.7, 0.3,
                              b["counts"], b["probs"], b["tokens"], b["loss"], ws)
        capi.cap_router_grad(6000, 6, 96, d["logits"], d["idx"], d["keep"], d["w"], d["d_w"], d["mask"], d["offs"], S,
                             b["counts"], b["tokens"], 0.7, 0.3, None, capi.CAP_DTYPE_F32, out)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    first = d["logits"].clone()
    for i in range(4):
        d["logits"].copy_(first * (1 + 0.1 * i))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*b.values(), out)]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (*b.values(), out)))


def test_offsets_past_32_bits():
    """2.2e9 logits: the last tokens' rows and the totals."""
    T, E, k = (1 << 23) + 5, 256, 2
    x = torch.zeros((T, E), device="cuda")
    x[-4:] = torch.randn((4, E), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    idx = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    idx[:, 1] = 1
    offs = torch.tensor([0, T - 4, T], dtype=torch.int32, device="cuda")
    counts = torch.empty((2, E), dtype=torch.int32, device="cuda")
    probs, tokens, loss = torch.empty((2, E), device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
    ws = torch.empty(capi.cap_workspace_size(capi.CAP_OP_BALANCE_LOSS, capi.Topology(E=E, T=T), max_rows=2),
                     dtype=torch.uint8, device="cuda")
    capi.cap_balance_loss(T, k, E, x, idx, None, None, offs, 2, 1.0, 0.0, counts, probs, tokens, loss, ws)
    out = torch.empty((T, E), device="cuda")
    capi.cap_router_grad(T, k, E, x, idx, None, None, None, None, offs, 2, counts, tokens, 1.0, 0.0, None,
                         capi.CAP_DTYPE_F32, out)
    torch.cuda.synchronize()
    assert tokens.tolist() == [T - 4, 4, 2, T] and counts[:, :3].tolist() == [[T - 4, T - 4, 0], [4, 4, 0]]
    tail = x[-4:].cpu().numpy()
    ref = R.balance64(tail, np.tile([[0, 1]], (4, 1)).astype(np.int32))
    _near(probs[1].cpu().numpy(), ref["probs"][0], TOL, "probs of the last sequence")
    _near(probs[0].cpu().numpy(), np.full(E, 1 / E), TOL, "probs of the first")
    want = 0.5 * R.grad64(tail, np.tile([[0, 1]], (4, 1)).astype(np.int32), None, None, None, None, None, 1.0, 0.0)
    _near(out[-4:].cpu().numpy(), want, TOL, "rows of the last tokens")


def test_pruned_routing_of_the_layer():
    """On the framework's own routing outputs."""
    from workloads import generator as gen
    cfg = gen.CONFIGS["c2"]
    T = 4096
    er, el = gen.sequential_placement(cfg)
    er, el = torch.from_numpy(er).cuda(), torch.from_numpy(el).cuda()
    topo = capi.make_topology(cfg.E, cfg.R, cfg.ranks_per_node, T, cfg.k, er, el)
    logits = gen.logits(cfg)[:T]
    x = torch.from_numpy(logits).cuda()
    idx = torch.empty((T, cfg.k), dtype=torch.int32, device="cuda")
    w, keep = torch.empty((T, cfg.k), device="cuda"), torch.empty((T, cfg.k), dtype=torch.uint8, device="cuda")
    dst = torch.empty(T, dtype=torch.int64, device="cuda")
    capi.cap_route_prune(topo, x, 0.3, idx, w, keep, dst)
    d_w = np.random.default_rng(2).standard_normal((T, cfg.k)).astype(np.float32)
    c = dict(logits=logits, idx=idx.cpu().numpy(), keep=keep.cpu().numpy(), w=w.cpu().numpy(), d_w=d_w, mask=None,
             offsets=_ragged(T, 8, 9))
    d, o, S = _forward(c)
    _check_forward(c, o)
    assert o["counts"].sum().item() == keep.sum().item()
    want = R.grad64(c["logits"], c["idx"], c["keep"], c["w"], c["d_w"], None, c["offsets"], 0.7, 0.3)
    _near(_backward(c, d, o, S).cpu().numpy(), want, TOL, "d_logits")
