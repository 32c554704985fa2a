"""rotary against the formula in 64 bits: axes, formats of positions, far positions, partly turned heads, strides.

Tolerance: the angle's sine and cosine are right to 2^-21 (an angle rounded to fp32 within half a turn, 2^-24 of it, and the
functions' own last bits), the products and their sum to 2^-22 of |x1| + |x2|, and the result is rounded once: u |y| + 2^-20 (|x1| +
|x2|), u half a step of the format; fp16 below 2^-14 has steps of 2^-24."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _ag():
    from paper_2309_16669_amd import autograd
    return autograd


def _reference(x, positions, freqs, sections, interleaved, sign=1):
    """positions [axes, P] on tokens flattened to T = multiples of P."""
    x = x.detach().cpu().double()
    flat = x.reshape(-1, *x.shape[-2:])
    T, m = flat.shape[0], freqs.numel()
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    # (angles in the long form: 2^40 times a frequency has more bits than a double)
    pos = positions.cpu().reshape(len(sections), -1).numpy().astype(np.longdouble)
    angle = sign * pos[axis].T * freqs.cpu().numpy().astype(np.longdouble)
    cos, sin = (torch.from_numpy(f(angle).astype(np.float64)).repeat(T // angle.shape[0], 1)[:, None] for f in (np.cos, np.sin))
    a, b = (flat[..., 0:2 * m:2], flat[..., 1:2 * m:2]) if interleaved else (flat[..., :m], flat[..., m:2 * m])
    y, size = flat.clone(), torch.zeros_like(flat)
    at = (slice(0, 2 * m, 2), slice(1, 2 * m, 2)) if interleaved else (slice(0, m), slice(m, 2 * m))
    y[..., at[0]], y[..., at[1]] = a * cos - b * sin, b * cos + a * sin
    size[..., at[0]] = size[..., at[1]] = a.abs() + b.abs()
    return y.view(x.shape), size.view(x.shape)


def _close(got, want, size):
    u = torch.finfo(got.dtype).eps / 2
    least = 2.0 ** -25 if got.dtype == torch.float16 else 0.0
    err = (got.detach().cpu().double() - want).abs()
    assert (err <= u * want.abs() + 2.0 ** -20 * size + least).all(), float((err - u * want.abs()).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("lead,Hq,Hk,d,sections,kind", [
    ((1,), 1, 1, 64, (32,), torch.int64), ((7,), 12, 0, 64, (32,), torch.int32), ((3, 50), 16, 2, 80, (16, 12, 12), torch.int32),
    ((2, 5, 33), 3, 3, 128, (10, 10, 4), torch.float32), ((1001,), 4, 1, 80, (8,), torch.int64), ((4, 600), 5, 5, 16, (8,), torch.int32),
    ((2, 40), 2, 1, 72, (9, 9, 9, 5), torch.int64), ((33,), 1, 1, 1024, (512,), torch.float32)], ids=str)
def test_turns_and_gradients(lead, Hq, Hk, d, sections, kind, interleaved, dtype):
    g = torch.Generator().manual_seed(1)
    q, dq = (torch.randn((*lead, Hq, d), generator=g).to(dtype).cuda() for _ in range(2))
    k, dk = (torch.randn((*lead, Hk, d), generator=g).to(dtype).cuda() for _ in range(2)) if Hk else (None, None)
    shape = lead[1:] or lead            # shared over the first axis, where there is more than one
    places = torch.randint(-3000, 70000, (len(sections), *shape), generator=g)
    places = (places.float() / 4 if kind == torch.float32 else places).to(kind).cuda()
    freqs = _ag().rotary_frequencies(sections, device="cuda")
    q.requires_grad_(True)
    if Hk:
        k.requires_grad_(True)
    one = len(sections) == 1
    out = _ag().rotary(q, k, places[0] if one else places, freqs, None if one else sections, interleaved)
    outs, ins, grads = ((out,), (q,), (dq,)) if k is None else (out, (q, k), (dq, dk))
    for y, x in zip(outs, ins):
        _close(y, *_reference(x, places, freqs, sections, interleaved))
    for y, x in zip(torch.autograd.grad(outs, ins, grads), grads):
        _close(y, *_reference(x, places, freqs, sections, interleaved, -1))


def test_far_positions():
    """10^9 + 1 and 2^40: the angle keeps every bit."""
    q = torch.randn((3, 1, 64), generator=torch.Generator().manual_seed(2)).half().cuda()
    freqs = _ag().rotary_frequencies(32, device="cuda")
    for first in (10 ** 9 + 1, 2 ** 40, -(2 ** 40) + 7):
        places = torch.arange(first, first + 3, device="cuda")
        _close(_ag().rotary(q, None, places, freqs), *_reference(q, places[None], freqs, (32,), False))


def test_strides_places_and_one_gradient():
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((2, 30, 8, 64), generator=g).to(torch.bfloat16).cuda()
    places, freqs = torch.arange(30, device="cuda"), _ag().rotary_frequencies(32, device="cuda")
    q, k = qkv[:, :, :4], qkv[:, :, 4:6]
    want = _ag().rotary(q.contiguous(), k.contiguous(), places, freqs)
    odd = torch.empty(q.numel() + 1, dtype=q.dtype, device="cuda")[1:].view(q.shape).copy_(q)
    for a, b in ((q, k), (q.transpose(2, 3).contiguous().transpose(2, 3), k), (odd, k)):
        assert all(torch.equal(x, y) for x, y in zip(_ag().rotary(a, b, places, freqs), want))
    # one tensor for all heads (stride 0), and places for each token
    same = q[:, :, :1].expand(2, 30, 4, 64)
    assert torch.equal(_ag().rotary(same, None, places.expand(2, 30), freqs), _ag().rotary(same.contiguous(), None, places, freqs))
    leaf = qkv.clone().requires_grad_(True)
    y, z = _ag().rotary(leaf[:, :, :4], leaf[:, :, 4:6], places, freqs)
    z.float().sum().backward()          # the queries' gradient is absent
    ref, size = _reference(torch.ones_like(k), places[None], freqs, (32,), False, -1)
    _close(leaf.grad[:, :, 4:6], ref, size)
    assert not leaf.grad[:, :, :4].any() and not leaf.grad[:, :, 6:].any()
    assert _ag().rotary(q[:, :0], None, places[:0], freqs).shape == (2, 0, 4, 64)


def test_binding_in_place_and_on_a_stream():
    import paper_2309_16669_amd as av
    q = torch.randn((40, 3, 80), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    places, freqs = torch.arange(40, device="cuda", dtype=torch.int32)[None], _ag().rotary_frequencies(24, device="cuda")
    want = _ag().rotary(q, None, places[0], freqs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    av.rotary(q, None, places, freqs, (24,), q, None, stream=s)
    s.synchronize()
    assert torch.equal(q, want)


def test_infinities_stay_in_their_pair():
    q = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    q[0, 0, 3], q[0, 0, 40] = float("inf"), float("nan")
    y = _ag().rotary(q, None, torch.tensor([5], device="cuda"), _ag().rotary_frequencies(32, device="cuda"))[0, 0]
    hit = {3, 35, 8, 40}
    assert all(bool(torch.isfinite(y[i])) == (i not in hit) for i in range(64))


def test_graph_and_second_derivative():
    q, k = (torch.randn((50, h, 64), generator=torch.Generator().manual_seed(5)).half().cuda() for h in (4, 2))
    places, freqs = torch.arange(50, device="cuda"), _ag().rotary_frequencies((12, 10, 10), device="cuda")
    places = torch.stack([places, places + 3, places * 2])
    _ag().rotary(q, k, places, freqs, (12, 10, 10))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _ag().rotary(q, k, places, freqs, (12, 10, 10))
    for n in range(3):
        places.add_(n * 17)
        q.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, _ag().rotary(q, k, places, freqs, (12, 10, 10))))
    q.requires_grad_(True)
    y = _ag().rotary(q, None, places, freqs, (12, 10, 10))
    w = torch.ones_like(y).requires_grad_(True)
    (g,) = torch.autograd.grad(y, (q,), w, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        g.float().sum().backward()


@pytest.mark.parametrize("native", [True, False])
def test_one_axis_of_positions_stacked(native, monkeypatch):
    if not native:
        import types
        monkeypatch.setattr(_ag(), "_native", types.SimpleNamespace(rotary=lambda *args: None))
    q = torch.randn((2, 30, 3, 64), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    places, freqs = torch.arange(7, 37, device="cuda"), _ag().rotary_frequencies(24, device="cuda")
    want = _ag().rotary(q, None, places, freqs)
    for given in (places, places[None], places.expand(2, 30), places.expand(1, 2, 30)):
        assert torch.equal(_ag().rotary(q, None, given, freqs, (24,)), want)


def test_no_head_on_one_side():
    """No key head: the queries turn, and nothing comes back beside them.  No query head beside keys: refused."""
    import paper_2309_16669_amd as av
    x, none = torch.randn((30, 3, 64), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda(), torch.zeros((30, 0, 64), dtype=torch.bfloat16, device="cuda")
    places, freqs = torch.arange(30, device="cuda"), _ag().rotary_frequencies(32, device="cuda")
    y, z = _ag().rotary(x, none, places, freqs)
    assert torch.equal(y, _ag().rotary(x, None, places, freqs)) and z.shape == none.shape
    with pytest.raises(av.AvionError):
        _ag().rotary(none, x, places, freqs)
