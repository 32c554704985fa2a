"""attention_ragged against a plain implementation in 64 bits: lengths, head layouts, formats, masks, strides, empty sequences,
every kernel behind it, and what it must not touch.

Tolerances.  u is half a step of the format (bf16 2^-8, fp16 2^-11).  With A = P |V| the forward is off by at most
u |O| (its own rounding) + u (A + |O|) (weights rounded before they meet V, and their sum over the rounded ones), and in the
backward, with dS rounded once, dV by u |dV| + u P^T |dO|, dQ by u |dQ| + scale (u |dS| + P e) |K| and dK alike, where e = |dO| (bound
of O) is what the rounded O leaves in delta.  Scores and dP are sums of d products in fp32: off by at most (d + 2) 2^-24 of the sum of
the magnitudes, which the weights take as a factor.  fp16 has no normal numbers below 2^-14: an absolute 2^-25 a rounded value (dV's
weights are held 2^8 times larger)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F16 = torch.bfloat16, torch.float16


def _ag():
    from paper_2309_16669_amd import autograd
    return autograd


def _offsets(lengths, device="cuda"):
    return torch.tensor([0] + list(torch.tensor(lengths).cumsum(0)) if lengths else [0], dtype=torch.int32, device=device)


def _inputs(nq, nk, Hq, Hk, d, dtype, seed=0, tail=(0, 0)):
    g = torch.Generator().manual_seed(seed)
    Tq, Tk = sum(nq) + tail[0], sum(nk) + tail[1]
    q, k, v, do = (torch.randn(s, generator=g).to(dtype).cuda() for s in ((Tq, Hq, d), (Tk, Hk, d), (Tk, Hk, d), (Tq, Hq, d)))
    return q, k, v, do


def _reference(q, k, v, do, nq, nk, scale, causal):
    """Results and their bounds, in 64 bits on the host."""
    u = torch.finfo(q.dtype).eps / 2
    least = 2.0 ** -25 if q.dtype == F16 else 0.0
    q, k, v, do = (t.detach().cpu().double() for t in (q, k, v, do))
    Hq, Hk, d = q.shape[1], k.shape[1], q.shape[2]
    G = Hq // Hk
    out = {n: torch.zeros_like(t) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    tol = {n: torch.zeros_like(t) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    a = b = 0
    fp = (d + 2) * 2.0 ** -24
    for m, n in zip(nq, nk):
        for h in range(Hq if m and n else 0):
            Q, K, V, D = q[a:a + m, h], k[b:b + n, h // G], v[b:b + n, h // G], do[a:a + m, h]
            s = scale * Q @ K.t()
            es = scale * fp * (Q.abs() @ K.abs().t()).amax(1, keepdim=True) + 2.0 ** -22 * (s.abs().amax(1, keepdim=True) + 1)
            if causal:
                see = torch.arange(n)[None] <= torch.arange(m)[:, None] + n - m
                s = torch.where(see, s, torch.full_like(s, -math.inf))
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
            p = p / p.sum(1, keepdim=True).clamp_min(1e-300)
            O, A = p @ V, p @ V.abs()
            tO = u * (2 * O.abs() + A) + 3 * es * A + least * (V.abs().sum(0) + 1)
            out["o"][a:a + m, h], tol["o"][a:a + m, h] = O, tO
            dp = D @ V.t()
            edp = fp * (D.abs() @ V.abs().t())
            delta = (p * dp).sum(1, keepdim=True)
            e = (D.abs() * tO).sum(1, keepdim=True) + fp * (D.abs() * A).sum(1, keepdim=True)
            ds = p * (dp - delta)
            eds = u * ds.abs() + p * (e + edp) + 3 * es * ds.abs() + least
            eds = eds + u * (p * e)
            if causal:
                eds = torch.where(see, eds, torch.zeros_like(eds))
            dq, dk, dv = scale * ds @ K, scale * ds.t() @ Q, p.t() @ D
            out["dq"][a:a + m, h] = dq
            tol["dq"][a:a + m, h] = u * dq.abs() + scale * eds @ K.abs() + least
            out["dk"][b:b + n, h // G] += dk
            tol["dk"][b:b + n, h // G] += scale * eds.t() @ Q.abs()
            out["dv"][b:b + n, h // G] += dv
            tol["dv"][b:b + n, h // G] += (p * (u + 3 * es) + least / 256).t() @ D.abs()
        a, b = a + m, b + n
    for n in ("dk", "dv"):
        tol[n] += u * out[n].abs() + least
    for n in tol:
        tol[n] = 1.01 * tol[n] + 1e-30
    return out, tol


def _compare(got, out, tol, names):
    for n in names:
        err = (got[n].detach().cpu().double() - out[n]).abs()
        bad = ~(err <= tol[n])
        assert not bad.any(), (n, int(bad.sum()), float((err / tol[n]).max()), bad.nonzero()[0].tolist())


def _check(nq, nk, Hq, Hk, d, dtype, causal, scale=None, seed=0):
    q, k, v, do = _inputs(nq, nk, Hq, Hk, d, dtype, seed)
    scale = 1 / math.sqrt(d) if scale is None else scale
    for t in (q, k, v):
        t.requires_grad_(True)
    oq = _offsets(nq)
    ok = None if nq == nk else _offsets(nk)
    o = _ag().attention_ragged(q, k, v, oq, ok, scale, causal)
    dq, dk, dv = torch.autograd.grad(o, (q, k, v), do)
    with torch.no_grad():
        assert torch.equal(o, _ag().attention_ragged(q, k, v, oq, ok, scale, causal))
    out, tol = _reference(q, k, v, do, nq, nk, scale, causal)
    _compare({"o": o, "dq": dq, "dk": dk, "dv": dv}, out, tol, ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hk,d", [(2, 2, 64), (4, 1, 80), (6, 2, 128)])
@pytest.mark.parametrize("lengths", [[1], [31, 32, 33], [5, 0, 64, 1, 65], [128, 129, 127], [200, 3, 257]], ids=str)
def test_same_lengths(lengths, Hq, Hk, d, dtype, causal):
    _check(lengths, lengths, Hq, Hk, d, dtype, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hq,Hk,d,dtype", [(3, 3, 64, BF), (8, 1, 64, F16), (16, 2, 80, BF), (5, 1, 128, F16), (2, 1, 128, BF)])
@pytest.mark.parametrize("nq,nk", [([1, 1, 1], [70, 1, 300]), ([7, 0, 40], [130, 20, 0]), ([90, 5], [30, 5]), ([1] * 70, list(range(70))),
                                   ([65, 300], [200, 301]), ([2, 1, 1], [700, 1300, 520])], ids=str)
def test_other_keys_than_queries(nq, nk, Hq, Hk, d, dtype, causal):
    _check(nq, nk, Hq, Hk, d, dtype, causal)


@pytest.mark.parametrize("d,dtype", [(64, BF), (80, F16), (128, BF)])
def test_single_tokens_in_chunks(d, dtype):
    nk = [2100, 255, 256, 257, 0, 5000]
    _check([1, 1, 1, 1, 1, 1], nk, 8, 2, d, dtype, True)
    _check([1, 2, 1, 0, 1, 20], nk, 4, 1, d, dtype, True)     # 80 rows: past one tile
    _check([1, 2, 1, 0, 1, 20], nk, 4, 1, d, dtype, False)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,dtype", [(64, F16), (80, BF), (128, BF)])
@pytest.mark.parametrize("nq,nk", [([1, 1, 300, 1, 0, 5, 40], [1100, 3000, 2100, 1, 700, 255, 700]), ([1] * 90, [256, 400, 300] * 30),
                                   ([1] * 60 + [200], [300] * 60 + [0])], ids=["mixed", "single", "long"])
def test_prompts_among_single_tokens(nq, nk, d, dtype, causal):
    _check(nq, nk, 4, 1, d, dtype, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hq,Hk,d,dtype,nq,nk", [
    (32, 32, 64, BF, [300, 129, 64, 1, 200] * 4, None), (32, 16, 128, F16, [260, 130, 7], [300, 130, 90]), (64, 32, 80, BF, [150] * 10, None),
    (12, 12, 64, F16, [300, 129, 64, 1, 600], None), (8, 8, 128, BF, [500, 700, 130], None), (20, 10, 80, F16, [513, 200, 140], [300, 900, 140]),
    (1, 1, 64, BF, [1100, 77], None), (4, 2, 128, F16, [700], [1000]),
    (40, 40, 80, BF, [300, 500, 130], None), (26, 13, 128, F16, [700, 300, 513], [700, 0, 600])], ids=str)
def test_every_cut(Hq, Hk, d, dtype, nq, nk, causal):
    """Whole blocks of 128 rows (from 512 of them), two groups of wavefronts (from 96, above 64 channels with smaller tiles from 256) and
    four."""
    _check(nq, nq if nk is None else nk, Hq, Hk, d, dtype, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,dtype", [(64, BF), (64, F16), (80, BF), (128, F16)], ids=str)
@pytest.mark.parametrize("nq,nk", [([1, 31, 32, 33, 63, 64, 65, 0, 5, 96], None), ([5, 40, 64, 1, 0, 33, 2], [9, 20, 64, 33, 12, 0, 70])], ids=str)
def test_short_sequences_whole(nq, nk, d, dtype, causal):
    """Up to 32, to 64 and above, mixed; fewer keys than queries, none on either side."""
    pad = [3] * 20          # short on average
    _check(nq + pad, (nq if nk is None else nk) + pad, 2, 2, d, dtype, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,dtype", [(64, F16), (80, BF), (80, F16)], ids=str)
def test_sequences_whole_up_to_128_tokens(d, dtype, causal):
    nq = [128, 127, 120, 97, 110, 125, 128]     # 119 on average
    _check(nq, nq, 3, 3, d, dtype, causal)
    _check(nq, nq[::-1], 3, 3, d, dtype, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("S", [1, 2, 7, 61, 62])
@pytest.mark.parametrize("same", [True, False])
def test_order_of_sequences(S, same, causal):
    """Up to 61 sequences begin by length: ties, and none on one side."""
    g = torch.Generator().manual_seed(S)
    nq = [150] * S if same else torch.randint(0, 300, (S,), generator=g).tolist()
    nk = nq if same else torch.randint(0, 300, (S,), generator=g).tolist()
    if not same:
        nq[S // 2], nk[S // 3] = 0, 0
    _check(nq, nk, 2, 1, 64, BF, causal)


def test_many_sequences():
    g = torch.Generator().manual_seed(3)
    nq = torch.randint(0, 9, (5000,), generator=g).tolist()   # three steps of the search
    _check(nq, nq, 1, 1, 64, BF, True)


@pytest.mark.parametrize("scale", [0.02, 1.0, 4.0])
def test_scales(scale):
    _check([100, 200], [100, 200], 2, 1, 64, BF, True, scale)


@pytest.mark.parametrize("d", [64, 80, 128])
def test_growing_scores(d):
    """Keys that grow along the sequence: the running maximum rises again and again."""
    q, k, v, do = _inputs([160], [320], 4, 2, d, BF, 5)
    k = (k.float() * torch.linspace(0.1, 12, 320, device="cuda")[:, None, None]).to(BF)
    for t in (q, k, v):
        t.requires_grad_(True)
    o = _ag().attention_ragged(q, k, v, _offsets([160]), _offsets([320]), 0.5, False)
    g = torch.autograd.grad(o, (q, k, v), do)
    out, tol = _reference(q, k, v, do, [160], [320], 0.5, False)
    _compare(dict(zip(("o", "dq", "dk", "dv"), (o, *g))), out, tol, ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("single", [False, True])
def test_rows_of_no_sequence_and_neighbours(single):
    """Rows outside the offsets come out as zeros with zero gradients; what lies there, or in another sequence, reaches nothing."""
    nq, nk = ([1, 1, 1], [600, 300, 411]) if single else ([40, 70, 150], [40, 90, 150])
    q, k, v, do = _inputs(nq, nk, 4, 2, 64, BF, 1)
    pad = torch.full((9, 4, 64), math.nan, dtype=BF, device="cuda")
    wrap = lambda t: torch.cat([pad[:, :t.shape[1]], t, pad[:, :t.shape[1]]])   # noqa: E731
    shift = lambda n: _offsets(n) + 9   # noqa: E731
    with torch.no_grad():
        k2, v2, q2 = k.clone(), v.clone(), q.clone()
        a, b = nk[0], nk[0] + nk[1]
        k2[a:b], v2[a:b] = math.inf, math.nan
        q2[nq[0]:nq[0] + nq[1]] = math.nan
        do2 = do.clone()
        do2[nq[0]:nq[0] + nq[1]] = math.inf
    want = {}
    for name, args in (("clean", (q, k, v, do, _offsets(nq), _offsets(nk))),
                       ("dirty", (*(wrap(t) for t in (q2, k2, v2, do2)), shift(nq), shift(nk)))):
        x = [t.detach().clone().requires_grad_(True) for t in args[:3]]
        o = _ag().attention_ragged(*x, args[4], args[5], causal=True)
        want[name] = (o, *torch.autograd.grad(o, x, args[3]))
    for clean, dirty, n in zip(want["clean"], want["dirty"], (nq, nq, nk, nk)):
        assert not dirty[:9].any() and not dirty[-9:].any()
        inner = dirty[9:-9]
        for s in (slice(0, n[0]), slice(n[0] + n[1], None)):
            assert torch.equal(inner[s], clean[s])


def test_slices_of_a_projection_and_other_strides():
    nq = [33, 140]
    T, Hq, Hk, d = sum(nq), 4, 2, 64
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn((T, Hq + 2 * Hk, d), generator=g).to(BF).cuda()
    do = torch.randn((T, Hq, d), generator=g).to(BF).cuda()
    parts = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    results = []
    for make in (lambda t: t.clone(), lambda t: t, lambda t: t.transpose(0, 1).contiguous().transpose(0, 1),
                 lambda t: torch.empty(t.numel() + 1, dtype=BF, device="cuda")[1:].view(t.shape).copy_(t)):
        x = [make(t).detach().requires_grad_(True) for t in parts]
        o = _ag().attention_ragged(*x, _offsets(nq), causal=True)
        results.append((o, *torch.autograd.grad(o, x, do)))
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[0]))
    leaf = qkv.clone().requires_grad_(True)
    o = _ag().attention_ragged(leaf[:, :Hq], leaf[:, Hq:Hq + Hk], leaf[:, Hq + Hk:], _offsets(nq), causal=True)
    o.backward(do)
    assert torch.equal(leaf.grad, torch.cat(results[0][1:], 1))


def test_gradients_against_differences():
    nq, nk, d = [3, 6], [5, 6], 64
    q, k, v, do = (t.double() for t in _inputs(nq, nk, 2, 1, d, F16, 7))
    x = [t.to(F16).requires_grad_(True) for t in (q, k, v)]
    o = _ag().attention_ragged(*x, _offsets(nq), _offsets(nk), causal=True)
    got = torch.autograd.grad(o, x, do.to(F16))
    def value(*t):
        # the formula in 64 bits
        out, _ = _reference(*t, do, nq, nk, 1 / math.sqrt(d), True)
        return float((out["o"] * do.cpu()).sum())
    _, tol = _reference(*(t.to(F16) for t in (q, k, v)), do.to(F16), nq, nk, 1 / math.sqrt(d), True)
    base = [t.detach().double().cpu() for t in x]
    for i, (g, n) in enumerate(zip(got, ("dq", "dk", "dv"))):
        for at in ((0, 0, 0), (4, 0, 7), (8, g.shape[1] - 1, 63)):
            step = 1e-4
            hi, lo = [t.clone() for t in base], [t.clone() for t in base]
            hi[i][at] += step
            lo[i][at] -= step
            want = (value(*hi) - value(*lo)) / (2 * step)
            assert abs(float(g[at]) - want) <= float(tol[n][at]) + 1e-6, (n, at)


def test_binding_leaves_the_rest_alone_and_streams():
    """The C interface on another stream than the current one, workspace full of NaN, outputs as they are described."""
    import paper_2309_16669_amd as av
    nq, nk = [50, 1], [50, 400]
    q, k, v, do = _inputs(nq, nk, 4, 2, 64, BF, 4)
    sizes = (51, 450, 2, 4, 2, 64)
    o, lse = torch.empty_like(q), torch.empty((4, 51), dtype=torch.float32, device="cuda")
    wf = torch.full((av.ragged_fwd_workspace_bytes(*sizes),), 255, dtype=torch.uint8, device="cuda")
    wb = torch.full((av.ragged_bwd_workspace_bytes(*sizes),), 255, dtype=torch.uint8, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    av.ragged_fwd(q, k, v, _offsets(nq), _offsets(nk), o, lse, 0.125, wf, True, s)
    av.ragged_bwd(q, k, v, _offsets(nq), _offsets(nk), o, lse, do, dq, dk, dv, 0.125, wb, True, s)
    torch.cuda.synchronize()
    out, tol = _reference(q, k, v, do, nq, nk, 0.125, True)
    _compare({"o": o, "dq": dq, "dk": dk, "dv": dv}, out, tol, ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("nq,nk", [([30, 100], [30, 100]), ([1, 1], [900, 1500])], ids=str)
def test_graph(nq, nk):
    q, k, v, do = _inputs(nq, nk, 4, 1, 64, BF, 6)
    for t in (q, k, v):
        t.requires_grad_(True)
    oq, ok = _offsets(nq), _offsets(nk)

    def step():
        o = _ag().attention_ragged(q, k, v, oq, ok, causal=True)
        return (o.detach(), *torch.autograd.grad(o, (q, k, v), do))

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
            for t, new in zip((q, k, v, do), _inputs(nq, nk, 4, 1, 64, BF, 20 + seed)):
                t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, step()))


def test_no_second_derivative():
    q, k, v, do = _inputs([8], [8], 1, 1, 64, BF)
    q.requires_grad_(True)
    o = _ag().attention_ragged(q, k, v, _offsets([8]))
    (g,) = torch.autograd.grad(o, (q,), do, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        g.float().sum().backward()


@pytest.mark.parametrize("S", [3, 70])
def test_offsets_outside_the_tensors(S):
    """Taken as the nearest place inside; decreasing ones write nowhere but in the outputs."""
    import paper_2309_16669_amd as av
    T, Hq, Hk, d = 500, 4, 2, 64
    q, k, v, do = _inputs([T], [T], Hq, Hk, d, BF, S)
    inside = [0] * (S - 2) + [40, 300, T]
    outside = [-7] * (S - 2) + [40, 300, 2 ** 31 - 1]
    guard = 64

    def run(offsets):
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        whole = {n: torch.full((T + 2 * guard, H, d), 7.0, dtype=BF, device="cuda") for n, H in (("o", Hq), ("dq", Hq), ("dk", Hk), ("dv", Hk))}
        y = {n: t[guard:-guard] for n, t in whole.items()}
        lse = torch.empty((Hq, T), dtype=torch.float32, device="cuda")
        space = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")   # noqa: E731
        av.ragged_fwd(q, k, v, off, off, y["o"], lse, 0.125, space(av.ragged_fwd_workspace_bytes(T, T, S, Hq, Hk, d)), True)
        av.ragged_bwd(q, k, v, off, off, y["o"], lse, do, y["dq"], y["dk"], y["dv"], 0.125, space(av.ragged_bwd_workspace_bytes(T, T, S, Hq, Hk, d)), True)
        for n, t in whole.items():
            assert (t[:guard] == 7).all() and (t[-guard:] == 7).all(), n
        return y

    a, b = run(inside), run(outside)
    assert all(torch.equal(a[n], b[n]) for n in a)
    g = torch.Generator().manual_seed(S)
    for _ in range(3):
        run(torch.randint(-50, 700, (S + 1,), generator=g).tolist())


def _many(S, kind, seed):
    """Queries and keys of S sequences."""
    g = torch.Generator().manual_seed(seed)
    if kind == "tokens":        # one behind a cache each
        return [1] * S, torch.randint(200, 420, (S,), generator=g).tolist()
    nq = torch.randint(0, 60 if kind != "blocks" else 190, (S,), generator=g).tolist()
    return nq, nq if kind != "other" else torch.randint(0, 60, (S,), generator=g).tolist()


def _some(S):
    """Sequences at the ends of what a step of the search leaves over (every 65th of 4031, 66th of 4157, ...), their neighbours, and some."""
    step = (S + 2 + 62) // 63
    ends = {i + k for i in range(step - 2, S, step) for k in (-1, 0, 1, 2)}
    return sorted(i for i in ends | {0, 1, S // 3, S // 2, S - 2, S - 1} | set(range(0, S, 97)) if 0 <= i < S)


@pytest.mark.parametrize("S,kind,Hq,Hk,d,dtype,causal", [
    (4031, "same", 1, 1, 64, BF, False), (4031, "same", 2, 1, 64, BF, True), (4031, "other", 1, 1, 64, F16, True), (4031, "other", 4, 1, 80, BF, False),
    (4031, "tokens", 4, 1, 64, BF, True), (4031, "blocks", 2, 1, 64, BF, True), (4031, "blocks", 1, 1, 64, F16, False),
    (4093, "same", 2, 2, 80, F16, True), (4093, "tokens", 8, 1, 128, BF, False), (4157, "other", 2, 1, 128, BF, True),
    (4157, "blocks", 2, 1, 80, BF, True), (4345, "same", 2, 1, 128, F16, True), (6050, "same", 1, 1, 64, BF, True), (6050, "tokens", 2, 1, 64, F16, True),
    (16384, "same", 1, 1, 64, BF, True), (16384, "other", 2, 1, 64, BF, False)], ids=str)
def test_every_sequence_of_many_is_its_own(S, kind, Hq, Hk, d, dtype, causal):
    """Numbers of sequences at which a wide step of the search leaves a single one: none may take its neighbour's tokens for its own."""
    nq, nk = _many(S, kind, S + d)
    g = torch.Generator("cuda").manual_seed(S)
    q, k, v, do = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in
                   ((sum(nq), Hq, d), (sum(nk), Hk, d), (sum(nk), Hk, d), (sum(nq), Hq, d)))
    for t in (q, k, v):
        t.requires_grad_(True)
    o = _ag().attention_ragged(q, k, v, _offsets(nq), None if nk is nq else _offsets(nk), causal=causal)
    dq, dk, dv = torch.autograd.grad(o, (q, k, v), do)
    with torch.no_grad():
        assert torch.equal(o, _ag().attention_ragged(q, k, v, _offsets(nq), None if nk is nq else _offsets(nk), causal=causal))
    bq, bk = _offsets(nq, "cpu").tolist(), _offsets(nk, "cpu").tolist()
    some = _some(S)
    rows = torch.cat([torch.arange(bq[i], bq[i + 1]) for i in some]).cuda()
    keys = torch.cat([torch.arange(bk[i], bk[i + 1]) for i in some]).cuda()
    out, tol = _reference(q[rows], k[keys], v[keys], do[rows], [nq[i] for i in some], [nk[i] for i in some], 1 / math.sqrt(d), causal)
    _compare({"o": o[rows], "dq": dq[rows], "dk": dk[keys], "dv": dv[keys]}, out, tol, ("o", "dq", "dk", "dv"))


def test_tens_of_thousands_of_heads_on_one():
    """32768 query heads, 2048 times the same 16, on one key head: O and dQ are those of the 16, dK and dV 2048 times theirs, up to the fp32
    sums' own roundings (each of less than 2^15 products of 16 rows, one after the other: 2^-9 of the magnitudes)."""
    nq, times, d = [40, 30], 2048, 64
    q, k, v, do = _inputs(nq, nq, 16, 1, d, BF, 8)
    x = [q.repeat(1, times, 1).requires_grad_(True), k.clone().requires_grad_(True), v.clone().requires_grad_(True)]
    o = _ag().attention_ragged(*x, _offsets(nq), causal=True)
    dq, dk, dv = torch.autograd.grad(o, x, do.repeat(1, times, 1))
    out, tol = _reference(q, k, v, do, nq, nq, 1 / math.sqrt(d), True)
    for first in (0, 16 * 1023, 16 * 2047):
        _compare({"o": o[:, first:first + 16], "dq": dq[:, first:first + 16]}, out, tol, ("o", "dq"))
    assert torch.equal(o, o[:, :16].repeat(1, times, 1)) and torch.equal(dq, dq[:, :16].repeat(1, times, 1))
    u = torch.finfo(BF).eps / 2
    for got, n in ((dk, "dk"), (dv, "dv")):
        # (what the bound of the 16 has beside the rounding of the result: at least u of the magnitudes that were summed)
        assert ((got.cpu().double() / times - out[n]).abs() <= tol[n] * (1 + 2.0 ** -9 / u)).all(), n
