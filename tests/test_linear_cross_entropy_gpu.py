"""linear_cross_entropy against the formula in 64 bits: sizes around every tile, formats, targets without a word, reductions, strides.

Tolerances, u half a step of the format (bf16 2^-8, fp16 2^-11).  Logits are fp32 sums of D exact products: off by at most
(D + 2) 2^-24 |x| |w|^T a logit, e; lse and loss by 2 e and a few steps of fp32 at their size and the sum's.  dz is rounded once, so
dx is off by u |dx| (its rounding) + scale (u + 3 e) |dz| |w|, with |dz| taken as p + onehot where a logit's error counts, and dw
alike; the sums over V or T add their own 2^-22 of the magnitudes.  fp16: dz is held 2^14 times larger, its least step is 2^-25
of 2^-14 of the largest row's."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F16 = torch.bfloat16, torch.float16


def _ag():
    from paper_2309_16669_amd import autograd
    return autograd


def _inputs(T, V, D, dtype, seed=0, none=0.2):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, D), generator=g).to(dtype).cuda()
    w = (torch.randn((V, D), generator=g) * 2 * D ** -0.5).to(dtype).cuda()
    t = torch.randint(0, V, (T,), generator=g)
    t[torch.rand((T,), generator=g) < none] = -100
    return x, w, t.cuda()


def _reference(x, w, t, scale, dloss, ignore=-100, where="cpu"):
    """Losses, dx, dw for the gradients dloss of the rows' losses, and their bounds, in 64 bits; on the host, or where it takes too long
    there."""
    u, f32 = torch.finfo(x.dtype).eps / 2, 2.0 ** -24
    least = 2.0 ** -39 if x.dtype == F16 else 0.0
    xd, wd, t = x.detach().to(where).double(), w.detach().to(where).double(), t.to(where).long()
    T, D = xd.shape
    V = wd.shape[0]
    has = (t >= 0) & (t < V) & (t != ignore)
    at = torch.where(has, t, torch.zeros_like(t))
    z = scale * xd @ wd.t()
    e = scale * (D + 2) * f32 * (xd.abs() @ wd.abs().t()).amax(1) + 4 * f32 * (z.abs().amax(1) + 1)
    lse = torch.logsumexp(z, 1)
    none, rows = torch.zeros(T, device=where).double(), torch.arange(T, device=where)
    loss = torch.where(has, lse - z[rows, at], none)
    loss_tol = torch.where(has, 2 * e + 8 * f32 * (lse.abs() + loss.abs() + 1), none)
    one = torch.zeros_like(z)
    one[rows, at] = 1
    p = torch.exp(z - lse[:, None])
    d = torch.where(has, dloss.to(where).double(), none)[:, None]
    dz, size = (p - one) * d, d.abs() * (p + one)
    edz = u * dz.abs() + (3 * e[:, None] + 4 * f32) * size + least * d.abs().max()
    dx, dw = scale * dz @ wd, scale * dz.t() @ xd
    dx_tol = u * dx.abs() + scale * (edz + 4 * f32 * dz.abs()) @ wd.abs() + least
    dw_tol = u * dw.abs() + scale * (edz + 4 * f32 * dz.abs()).t() @ xd.abs() + least
    if x.dtype == F16:      # results below its normal numbers
        dx_tol, dw_tol = dx_tol + 2.0 ** -25, dw_tol + 2.0 ** -25
    return tuple(a.cpu() for a in (loss, dx, dw)), tuple(a.cpu() for a in (loss_tol, 1.01 * dx_tol, 1.01 * dw_tol)), int(has.sum())


def _close(got, want, tol, name):
    err = (got.detach().cpu().double() - want).abs()
    assert (err <= tol).all(), (name, float((err / tol.clamp_min(1e-300)).max()), (err > tol).nonzero()[0].tolist())


def _check(x, w, t, scale=1.0, reduction="mean", dloss=None, where="cpu"):
    T = x.shape[0]
    x.requires_grad_(True)
    w.requires_grad_(True)
    out = _ag().linear_cross_entropy(x, w, t, scale, reduction=reduction)
    with torch.no_grad():
        assert torch.equal(out, _ag().linear_cross_entropy(x, w, t, scale, reduction=reduction))
    has = int(((t >= 0) & (t < w.shape[0])).sum())
    if reduction == "none":
        dloss = torch.linspace(-1, 2, T, device="cuda") if dloss is None else dloss
        given, rows = dloss, dloss
    else:
        given = torch.tensor(3.0, device="cuda")
        rows = torch.full((T,), 3.0 / max(1, has) if reduction == "mean" else 3.0)
    dx, dw = torch.autograd.grad(out, (x, w), given)
    (loss, rx, rw), (loss_tol, tx, tw), n = _reference(x, w, t, scale, rows, where=where)
    assert n == has
    if reduction == "none":
        _close(out, loss, loss_tol, "loss")
        assert not out[~((t >= 0) & (t < w.shape[0]))].any()
    else:
        by = max(1, n) if reduction == "mean" else 1
        _close(out, loss.sum() / by, loss_tol.sum() / by + 2.0 ** -23 * loss.sum() / by, "loss")
    _close(dx, rx, tx, "dx")
    _close(dw, rw, tw, "dw")


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("T,V,D", [(1, 1, 8), (1, 130, 64), (5, 1000, 72), (32, 129, 128), (33, 127, 8), (128, 257, 200), (129, 64, 776),
                                   (300, 1001, 64), (1000, 77, 136), (900, 5003, 72)], ids=str)
def test_sizes(T, V, D, reduction, dtype):
    _check(*_inputs(T, V, D, dtype, none=0.2 if T > 1 else 0.0), reduction=reduction)


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("T,V", [(4100, 4099), (5000, 4801)])
def test_large_tiles(T, V, dtype):
    """In the forward, and in dz from 23.5 million logits on."""
    _check(*_inputs(T, V, 72, dtype))


@pytest.mark.parametrize("T,V,D,dtype", [(4000, 4200, 2056, BF), (300, 60000, 1104, F16), (3000, 270, 4104, BF), (213, 30000, 72, BF),
                                         (20000, 100, 136, F16)], ids=str)
def test_gradients_of_large_tiles_and_ranges(T, V, D, dtype):
    """256 x 256 tiles in the gradients, whole and cut along K on either side; 128 x 128 ones cut many times."""
    _check(*_inputs(T, V, D, dtype), where="cuda")


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
def test_vocabulary_in_pieces(dtype, monkeypatch):
    """T so large that a piece holds 256 columns would take hours here; the sizes at which two pieces begin do not."""
    import paper_2309_16669_amd as av
    T, V, D = 150000, 4000, 8
    assert av.linear_ce_bwd_workspace_bytes(T, V, D) < T * V * 2 + (1 << 20) and av.linear_ce_bwd_workspace_bytes(T, V, D) > T * D * 4
    x, w, t = _inputs(T, V, D, dtype)
    x.requires_grad_(True)
    w.requires_grad_(True)
    out = _ag().linear_cross_entropy(x, w, t, reduction="none")
    g = torch.rand(T, device="cuda")
    dx, dw = torch.autograd.grad(out, (x, w), g)
    rows = torch.arange(0, T, 997)
    (loss, rx, _), (loss_tol, tx, _), _ = _reference(x[rows.cuda()], w, t[rows.cuda()], 1.0, g[rows.cuda()])
    _close(out[rows.cuda()], loss, loss_tol, "loss")
    _close(dx[rows.cuda()], rx, tx + (2.0 ** -39 if dtype == F16 else 0.0) * 4000, "dx")
    # dw of all rows: by blocks
    want, tol = 0, 0
    for i in range(0, T, 15000):
        (_, _, a), (_, _, b), _ = _reference(x[i:i + 15000], w, t[i:i + 15000], 1.0, g[i:i + 15000])
        want, tol = want + a, tol + b
    _close(dw, want, tol, "dw")


@pytest.mark.parametrize("scale", [0.01, 14.3, 100.0])
def test_pairs(scale):
    """A contrastive batch: unit rows, the logits far apart."""
    g = torch.Generator().manual_seed(1)
    a, b = (torch.nn.functional.normalize(torch.randn((500, 64), generator=g)) for _ in range(2))
    x, w = torch.nn.functional.normalize(a + b).to(BF).cuda(), b.to(BF).cuda()
    _check(x, w, torch.arange(500, device="cuda"), scale)


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_no_target_at_all(reduction):
    x, w, _ = _inputs(40, 50, 64, BF)
    x.requires_grad_(True)
    w.requires_grad_(True)
    t = torch.tensor([-100, -1, 50, 1 << 40] * 10, device="cuda")
    out = _ag().linear_cross_entropy(x, w, t, reduction=reduction)
    assert not out.any()
    assert not any(g.any() for g in torch.autograd.grad(out.sum(), (x, w)))


def test_ignored_index_int32_and_rows_of_nan():
    """An index inside the vocabulary can be the ignored one; what stands in a row without a target reaches nothing."""
    x, w, t = _inputs(70, 90, 64, BF, none=0.0)
    t[::3] = 7
    y = x.clone()
    y[t == 7] = float("nan")
    results = []
    for a, targets in ((x, torch.where(t == 7, -5, t)), (y, t), (y, t.int())):
        a, b = a.detach().clone().requires_grad_(True), w.detach().clone().requires_grad_(True)
        out = _ag().linear_cross_entropy(a, b, targets, ignore_index=7)
        results.append((out, *torch.autograd.grad(out, (a, b))))
    for r in results[1:]:
        assert torch.equal(r[0], results[0][0]) and torch.equal(r[1], results[0][1])
    # (dw multiplies those rows by zero: 0 * NaN is NaN, so only finite rows are compared)
    assert torch.isnan(results[1][2]).any() or torch.equal(results[1][2], results[0][2])


def test_strides_and_shapes():
    x, w, t = _inputs(60, 100, 64, BF)
    want = None
    for make in (lambda a: a.clone(), lambda a: torch.cat([a, a], 1)[:, :64], lambda a: a.t().contiguous().t(),
                 lambda a: torch.empty(a.numel() + 1, dtype=BF, device="cuda")[1:].view(a.shape).copy_(a)):
        a, b = make(x).detach().requires_grad_(True), make(w).detach().requires_grad_(True)
        out = _ag().linear_cross_entropy(a, b, t)
        got = (out, *torch.autograd.grad(out, (a, b)))
        want = want or got
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    a = x.view(3, 20, 64).detach().requires_grad_(True)
    out = _ag().linear_cross_entropy(a, w, t.view(3, 20), reduction="none")
    assert out.shape == (3, 20)
    out.sum().backward()
    assert a.grad.shape == a.shape
    # only one of the two wants a gradient
    b = w.detach().requires_grad_(True)
    _ag().linear_cross_entropy(x, b, t).backward()
    assert torch.equal(b.grad, want[2])
    assert not _ag().linear_cross_entropy(x[:0], w, t[:0]).any()


def test_gradient_against_differences():
    x, w, t = _inputs(6, 40, 16, F16, none=0.0)
    x.requires_grad_(True)
    w.requires_grad_(True)
    dx, dw = torch.autograd.grad(_ag().linear_cross_entropy(x, w, t, 2.0, reduction="sum"), (x, w))
    one = torch.ones(6)
    _, (_, tx, tw), _ = _reference(x, w, t, 2.0, one)
    base = [a.detach().cpu().double() for a in (x, w)]

    def value(a, b):
        z = 2.0 * a @ b.t()
        return float((torch.logsumexp(z, 1) - z[torch.arange(6), t.cpu()]).sum())

    for i, (g, tol) in enumerate(((dx, tx), (dw, tw))):
        for at in ((0, 0), (5, 15), (3, 7)):
            hi, lo = [a.clone() for a in base], [a.clone() for a in base]
            hi[i][at] += 1e-5
            lo[i][at] -= 1e-5
            assert abs(float(g[at]) - (value(*hi) - value(*lo)) / 2e-5) <= float(tol[at]) + 1e-7


def test_small_gradients_keep_their_bits():
    """A loss scaled down until each row's gradient is below fp16's numbers, up again by the caller's scale of dloss."""
    x, w, t = _inputs(200, 3000, 64, F16)
    _check(x, w, t, reduction="none", dloss=torch.linspace(1e-7, 3e-7, 200, device="cuda") * 1e9)
    _check(x, w, t, reduction="none", dloss=torch.zeros(200, device="cuda"))


def test_binding_on_a_stream_with_dirty_workspace():
    import paper_2309_16669_amd as av
    x, w, t = _inputs(100, 300, 72, BF)
    f = [torch.empty(s, dtype=torch.float32, device="cuda") for s in ((100,), (100,), (2,))]
    wf = torch.full((av.linear_ce_fwd_workspace_bytes(100, 300, 72),), 255, dtype=torch.uint8, device="cuda")
    wb = torch.full((av.linear_ce_bwd_workspace_bytes(100, 300, 72),), 255, dtype=torch.uint8, device="cuda")
    dx, dw, g = torch.empty_like(x), torch.empty_like(w), torch.tensor(1.0, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    av.linear_ce_fwd(x, w, t, f[0], f[1], f[2], 1.0, -100, wf, True, s)
    av.linear_ce_bwd(x, w, t, f[1], g, f[2], dx, dw, 1.0, -100, wb, True, s)
    torch.cuda.synchronize()
    n = int((t >= 0).sum())
    assert int(f[2][1]) == n
    (loss, rx, rw), (tl, tx, tw), _ = _reference(x, w, t, 1.0, torch.full((100,), 1 / n))
    for got, want, tol in ((f[0], loss, tl), (dx, rx, tx), (dw, rw, tw)):
        _close(got, want, tol, "binding")


def test_graph():
    x, w, t = _inputs(100, 500, 64, BF)
    x.requires_grad_(True)
    w.requires_grad_(True)

    def step():
        loss = _ag().linear_cross_entropy(x, w, t)
        return (loss.detach(), *torch.autograd.grad(loss, (x, w)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in range(3):
        with torch.no_grad():
            for a, b in zip((x, w, t), _inputs(100, 500, 64, BF, 30 + seed)):
                a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, step()))


def test_no_second_derivative():
    x, w, t = _inputs(8, 20, 64, BF)
    x.requires_grad_(True)
    (g,) = torch.autograd.grad(_ag().linear_cross_entropy(x, w, t), (x,), create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        g.float().sum().backward()


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
def test_what_a_row_without_a_target_holds_reaches_no_gradient(dtype):
    """Large finite numbers in such rows, an ignored index inside the vocabulary, int32: the bits of dw and dx of rows of zeros.  NaN and
    infinity are multiplied by zero for dw, and show there."""
    x, w, t = _inputs(70, 90, 64, dtype, none=0.0)
    t[::3] = 7
    none = t == 7
    results = []
    for held, targets in ((0.0, t), (3e4, t), (-6e4, t.int()), (1.0, torch.where(none, -5, t)), (2.0, torch.where(none, 90, t).int())):
        a, b = torch.where(none[:, None], torch.full_like(x, held), x).requires_grad_(True), w.detach().clone().requires_grad_(True)
        for reduction in ("mean", "none"):
            out = _ag().linear_cross_entropy(a, b, targets, ignore_index=7, reduction=reduction)
            results.append((out, *torch.autograd.grad(out, (a, b), torch.ones_like(out))))
    for r, want in zip(results[2:], results[:2] * 4, strict=True):
        assert all(torch.equal(p, q) for p, q in zip(r, want, strict=True))
    assert not results[0][1][none].any() and results[0][2].isfinite().all() and results[0][2].any()
    for held in (float("nan"), float("inf")):
        a, b = torch.where(none[:, None], torch.full_like(x, held), x).requires_grad_(True), w.detach().clone().requires_grad_(True)
        out = _ag().linear_cross_entropy(a, b, t, ignore_index=7)
        dx, dw = torch.autograd.grad(out, (a, b))
        assert torch.equal(out, results[0][0]) and torch.equal(dx, results[0][1]) and dw.isnan().all()


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("given", [float("inf"), float("-inf"), float("nan")])
def test_a_gradient_that_is_no_finite_number_makes_all_of_them_nan(given, reduction, dtype):
    """As the contract says: a loss scale that has overflowed cannot leave some gradients looking sound."""
    x, w, t = _inputs(70, 300, 64, dtype)
    t[0] = 5
    x.requires_grad_(True)
    w.requires_grad_(True)
    out = _ag().linear_cross_entropy(x, w, t, reduction=reduction)
    dloss = torch.ones_like(out)
    if reduction == "none":
        dloss[0] = given
    else:
        dloss.fill_(given)
    assert all(g.isnan().all() for g in torch.autograd.grad(out, (x, w), dloss))
