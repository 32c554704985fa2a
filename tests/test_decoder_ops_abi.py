"""Rotary positions, ragged attention and the loss over a vocabulary: what the C entry points and the front end refuse, before
anything is launched, and the sizes of their workspaces.  Runs without a GPU."""
import ctypes

import pytest

import paper_2309_16669_amd as av

P = 0x1000          # aligned, never dereferenced on these paths
f = ctypes.c_float
INF, NAN = float("inf"), float("nan")


def _rotary(q=P, k=P, positions=P, freqs=P, yq=P * 2, yk=P * 3, T=8, P_=8, Hq=4, Hk=2, d=64, pairs=32, sections=(32,), rs_q=256, rs_k=128, flags=0):
    c = None if sections is None else (ctypes.c_int * max(1, len(sections)))(*sections)
    return av.load_library().avion_rotary(q, k, positions, freqs, yq, yk, T, P_, Hq, Hk, d, pairs, c, 0 if sections is None else len(sections),
                                          rs_q, rs_k, flags, None)


def _ragged_fwd(q=P, k=P, v=P, oq=P, ok=P, o=P, lse=P, Tq=8, Tk=8, S=2, Hq=4, Hk=2, d=64, rs_q=256, rs_k=128, rs_v=128, scale=0.125, flags=0,
                ws=P, n=1 << 40):
    return av.load_library().avion_ragged_fwd(q, k, v, oq, ok, o, lse, Tq, Tk, S, Hq, Hk, d, rs_q, rs_k, rs_v, f(scale), flags, ws, n, None)


def _ragged_bwd(q=P, k=P, v=P, oq=P, ok=P, o=P, lse=P, dO=P, dq=P, dk=P, dv=P, Tq=8, Tk=8, S=2, Hq=4, Hk=2, d=64, rs_q=256, rs_k=128, rs_v=128,
                scale=0.125, flags=0, ws=P, n=1 << 40):
    return av.load_library().avion_ragged_bwd(q, k, v, oq, ok, o, lse, dO, dq, dk, dv, Tq, Tk, S, Hq, Hk, d, rs_q, rs_k, rs_v, f(scale), flags,
                                              ws, n, None)


def _ce_fwd(x=P, w=P, t=P, loss=P, lse=P, total=P, T=8, V=10, D=64, rs_x=64, rs_w=64, scale=1.0, ignore=-100, flags=0, ws=P, n=1 << 40):
    return av.load_library().avion_linear_ce_fwd(x, w, t, loss, lse, total, T, V, D, rs_x, rs_w, f(scale), ignore, flags, ws, n, None)


def _ce_bwd(x=P, w=P, t=P, lse=P, dloss=P, total=P, dx=P, dw=P, T=8, V=10, D=64, rs_x=64, rs_w=64, scale=1.0, ignore=-100, flags=0, ws=P,
            n=1 << 40):
    return av.load_library().avion_linear_ce_bwd(x, w, t, lse, dloss, total, dx, dw, T, V, D, rs_x, rs_w, f(scale), ignore, flags, ws, n, None)


ONE, MEAN = av.FLAG_ONE_GRADIENT, av.FLAG_MEAN
SHAPES = [(dict(Tq=-1), av.EINVAL), (dict(Tk=-1), av.EINVAL), (dict(S=-1), av.EINVAL), (dict(Hq=0), av.EINVAL), (dict(Hk=0), av.EINVAL),
          (dict(Hk=3), av.EINVAL), (dict(d=0), av.EINVAL), (dict(scale=0.0), av.EINVAL), (dict(scale=-1.0), av.EINVAL), (dict(scale=NAN), av.EINVAL),
          (dict(scale=INF), av.EINVAL), (dict(scale=1e-30), av.EINVAL), (dict(flags=4), av.EINVAL), (dict(flags=1 << 20), av.EINVAL),
          (dict(d=72, rs_q=288, rs_k=144, rs_v=144), av.EUNSUPPORTED), (dict(d=96, rs_q=384, rs_k=192, rs_v=192), av.EUNSUPPORTED),
          (dict(Tq=(1 << 28) + 1), av.EUNSUPPORTED), (dict(Tk=(1 << 28) + 1), av.EUNSUPPORTED), (dict(S=(1 << 20) + 1), av.EUNSUPPORTED),
          (dict(S=1 << 20, Hq=32, Hk=32, rs_q=2048, rs_k=2048, rs_v=2048), av.EUNSUPPORTED),
          (dict(Tq=1 << 28, Hq=16), av.EUNSUPPORTED), (dict(rs_q=255), av.EINVAL), (dict(rs_k=64), av.EINVAL), (dict(rs_v=127), av.EINVAL),
          (dict(rs_q=260), av.EUNSUPPORTED), (dict(rs_v=(1 << 23) + 8), av.EUNSUPPORTED), (dict(q=None), av.EINVAL), (dict(k=None), av.EINVAL),
          (dict(v=None), av.EINVAL), (dict(oq=None), av.EINVAL), (dict(ok=None), av.EINVAL), (dict(o=None), av.EINVAL), (dict(lse=None), av.EINVAL),
          (dict(q=P + 8), av.EUNSUPPORTED), (dict(k=P + 2), av.EUNSUPPORTED), (dict(oq=P + 2), av.EUNSUPPORTED), (dict(lse=P + 2), av.EUNSUPPORTED),
          (dict(o=P + 8), av.EUNSUPPORTED)]
LOSS = [(dict(T=-1), av.EINVAL), (dict(V=0), av.EINVAL), (dict(D=0), av.EINVAL), (dict(scale=0.0), av.EINVAL), (dict(scale=-1.0), av.EINVAL),
        (dict(scale=NAN), av.EINVAL), (dict(scale=INF), av.EINVAL), (dict(flags=2), av.EINVAL), (dict(x=None), av.EINVAL), (dict(w=None), av.EINVAL),
        (dict(t=None), av.EINVAL), (dict(lse=None), av.EINVAL), (dict(rs_x=56), av.EINVAL), (dict(rs_w=63), av.EINVAL),
        (dict(D=60, rs_x=64, rs_w=64), av.EUNSUPPORTED), (dict(D=65544, rs_x=65544, rs_w=65544), av.EUNSUPPORTED),
        (dict(T=1 << 28), av.EUNSUPPORTED), (dict(V=(1 << 28) + 1), av.EUNSUPPORTED), (dict(rs_x=68), av.EUNSUPPORTED),
        (dict(rs_w=(1 << 20) + 8), av.EUNSUPPORTED), (dict(x=P + 8), av.EUNSUPPORTED), (dict(w=P + 2), av.EUNSUPPORTED), (dict(t=P + 4), av.EUNSUPPORTED),
        (dict(t=P + 2, flags=av.FLAG_TOKENS_I32), av.EUNSUPPORTED), (dict(lse=P + 2), av.EUNSUPPORTED), (dict(total=P + 1), av.EUNSUPPORTED),
        (dict(ws=None), av.EWORKSPACE), (dict(ws=P + 16), av.EWORKSPACE), (dict(n=255), av.EWORKSPACE)]
CASES = [
    (_rotary, [(dict(T=-1), av.EINVAL), (dict(P_=0), av.EINVAL), (dict(P_=3), av.EINVAL), (dict(Hq=0), av.EINVAL), (dict(Hk=-1), av.EINVAL),
               (dict(d=0), av.EINVAL), (dict(pairs=0), av.EINVAL), (dict(pairs=40, sections=(40,)), av.EINVAL), (dict(sections=None), av.EINVAL),
               (dict(sections=(16, 8)), av.EINVAL), (dict(sections=(40, -8)), av.EINVAL), (dict(rs_q=248), av.EINVAL), (dict(rs_k=64), av.EINVAL),
               (dict(flags=2), av.EINVAL), (dict(flags=av.FLAG_TOKENS_I32 | av.FLAG_POSITIONS_F32), av.EINVAL), (dict(q=None), av.EINVAL),
               (dict(k=None), av.EINVAL), (dict(yq=None), av.EINVAL), (dict(yk=None), av.EINVAL), (dict(positions=None), av.EINVAL),
               (dict(freqs=None), av.EINVAL), (dict(q=P * 2, rs_q=512), av.EINVAL), (dict(sections=(8, 8, 8, 4, 4)), av.EUNSUPPORTED),
               (dict(d=68, rs_q=512, rs_k=512), av.EUNSUPPORTED), (dict(pairs=20, sections=(20,)), av.EUNSUPPORTED), (dict(rs_q=260), av.EUNSUPPORTED),
               (dict(d=4104, rs_q=1 << 20, rs_k=1 << 20), av.EUNSUPPORTED), (dict(T=1 << 27, P_=1 << 27), av.EUNSUPPORTED), (dict(q=P + 8), av.EUNSUPPORTED),
               (dict(yk=P + 8), av.EUNSUPPORTED), (dict(positions=P + 4), av.EUNSUPPORTED), (dict(freqs=P + 2), av.EUNSUPPORTED),
               (dict(T=0, q=None, yq=None), av.OK)]),
    (_ragged_fwd, SHAPES + [(dict(Tq=0, q=None, o=None, lse=None), av.OK),
                            (dict(Tq=2, Tk=2000, ws=None), av.EWORKSPACE), (dict(Tq=2, Tk=2000, ws=P + 128), av.EWORKSPACE),
                            (dict(Tq=2, Tk=2000, n=1000), av.EWORKSPACE)]),
    (_ragged_bwd, SHAPES + [(dict(dO=None), av.EINVAL), (dict(dq=None), av.EINVAL), (dict(dk=None), av.EINVAL), (dict(dv=None), av.EINVAL),
                            (dict(dO=P + 8), av.EUNSUPPORTED), (dict(dk=P + 4), av.EUNSUPPORTED), (dict(ws=None), av.EWORKSPACE),
                            (dict(ws=P + 64), av.EWORKSPACE), (dict(n=256), av.EWORKSPACE)]),
    (_ce_fwd, LOSS + [(dict(loss=None, total=None), av.EINVAL), (dict(loss=P + 2), av.EUNSUPPORTED), (dict(flags=ONE), av.EINVAL),
                      (dict(T=0, x=None, t=None, lse=None, total=None), av.OK)]),
    (_ce_bwd, LOSS + [(dict(dloss=None), av.EINVAL), (dict(dx=None, dw=None), av.EINVAL), (dict(dx=P + 8), av.EUNSUPPORTED),
                      (dict(dw=P + 2), av.EUNSUPPORTED), (dict(flags=MEAN), av.EINVAL), (dict(flags=MEAN | ONE, total=None), av.EINVAL),
                      (dict(dloss=P + 2), av.EUNSUPPORTED)]),
]


@pytest.mark.parametrize("call,kwargs,code", [(c, k, r) for c, cases in CASES for k, r in cases],
                         ids=lambda v: getattr(v, "__name__", None) or str(v))
def test_refused_without_launching(call, kwargs, code):
    assert call(**kwargs) == code


def test_workspace_sizes():
    fwd, bwd = av.ragged_fwd_workspace_bytes, av.ragged_bwd_workspace_bytes
    assert fwd(8, 8, 2, 4, 3, 64) == 0 and bwd(8, 8, 2, 4, 2, 96) == 0 and fwd(-1, 8, 2, 4, 2, 64) == 0
    assert fwd(4000, 4000, 9, 8, 8, 64) == 256          # nothing but whole sequences
    assert fwd(1, 10000, 1, 8, 2, 128) >= (10000 // 256) * 2 * 32 * 128 * 4
    # two floats a query and head, each sequence on a multiple of 64; planes only where the heads of a key head are dealt out
    assert 8 * 2 * 4000 * 4 <= bwd(4000, 4000, 9, 8, 8, 64) <= 8 * 2 * (4000 + 64 * 12) * 4 + 256
    for T in (0, 1, 1000):          # any sizes that can be asked for, without a crash
        for S in (0, 1, 7):
            for H in ((1, 1), (8, 1)):
                assert fwd(T, T, S, *H, 64) >= 256 and bwd(T, T, S, *H, 64) % 256 == 0 and fwd(0, T, S, *H, 80) >= 256
    ce_f, ce_b = av.linear_ce_fwd_workspace_bytes, av.linear_ce_bwd_workspace_bytes
    assert ce_f(8, 10, 60) == 0 and ce_b(8, 0, 64) == 0 and ce_f(0, 1, 8) >= 256 and ce_b(0, 1, 8) >= 256
    assert ce_f(16384, 50000, 768) < 16384 * 50000 // 256       # no logits
    assert ce_b(16384, 50000, 768) < (1 << 30) + 16384 * (768 * 4 + 12) + (1 << 20)
    assert ce_b((1 << 28) - 1, 1 << 28, 8) > 1 << 36                  # in size_t throughout


@pytest.mark.parametrize("last,first", [
    (dict(Hq=64, Tq=1 << 24), dict(Hq=64, Tq=(1 << 24) + 1)), (dict(Hq=1 << 16, Tq=1 << 14), dict(Hq=1 << 16, Tq=(1 << 14) + 1)),
    (dict(Tq=1 << 28), dict(Tq=(1 << 28) + 1)), (dict(Tk=1 << 28), dict(Tk=(1 << 28) + 1)), (dict(S=1 << 20), dict(S=(1 << 20) + 1)),
    (dict(Hq=1 << 16), dict(Hq=(1 << 16) + 1)), (dict(Hq=1 << 16, d=128), dict(Hq=(1 << 16) + 1, d=128)),
    (dict(Hq=8, Hk=8, Tq=(1 << 27) - (1 << 15), Tk=(1 << 27) - (1 << 15) - 128 * 3 - 1, S=3), dict(Hq=8, Hk=8, Tq=1 << 27, Tk=1 << 27, S=3)),
    (dict(Hq=16, Hk=16, S=(1 << 20) - 512 - 1), dict(Hq=16, Hk=16, S=1 << 20))], ids=str)
def test_the_limits_of_ragged_sequences_are_the_documented_ones(last, first):
    """The last sizes that the contract gives, and the next ones; nothing is launched."""
    for call in (av.ragged_fwd_workspace_bytes, av.ragged_bwd_workspace_bytes):
        at = [call(*(dict(dict(Tq=64, Tk=64, S=1, Hq=1, Hk=1, d=64), **sizes).values())) for sizes in (last, first)]
        assert at[0] >= 256 and at[1] == 0


def test_the_front_end_refuses():
    import torch
    from paper_2309_16669_amd import autograd as ag
    bf = torch.bfloat16
    q, k = torch.zeros(6, 4, 64, dtype=bf), torch.zeros(6, 2, 64, dtype=bf)
    at, freqs = torch.arange(6), torch.ones(32)
    off = torch.tensor([0, 6], dtype=torch.int32)
    x, w, t = torch.zeros(5, 64, dtype=bf), torch.zeros(9, 64, dtype=bf), torch.zeros(5, dtype=torch.int64)
    bad = [lambda: ag.rotary(q, k, at, freqs), lambda: ag.rotary(q, k[:3], at, freqs), lambda: ag.rotary(q, k, at[:4], freqs),
           lambda: ag.rotary(q, k, at, freqs, (16, 16)), lambda: ag.rotary(q[0], None, at[:0], freqs), lambda: ag.rotary(q.float(), None, at, freqs),
           lambda: ag.rotary(q, None, at.double(), freqs), lambda: ag.rotary(q, None, at, freqs[:16].double()),
           lambda: ag.attention_ragged(q, k, k, off), lambda: ag.attention_ragged(q, k, k, off.long()), lambda: ag.attention_ragged(q, k, k[:4], off),
           lambda: ag.attention_ragged(q, k, k, off, off[:1]), lambda: ag.attention_ragged(q[0], k, k, off), lambda: ag.attention_ragged(q, k.half(), k, off),
           lambda: ag.linear_cross_entropy(x, w, t), lambda: ag.linear_cross_entropy(x, w[:, :32], t), lambda: ag.linear_cross_entropy(x, w, t[:4]),
           lambda: ag.linear_cross_entropy(x, w, t, reduction="batch"), lambda: ag.linear_cross_entropy(x, w.half(), t),
           lambda: ag.linear_cross_entropy(x, w, t.short()), lambda: ag.linear_cross_entropy(x.float(), w.float(), t)]
    for call in bad:   # on the host, or in another format or shape
        with pytest.raises(ValueError):
            call()
    assert ag.rotary_frequencies((4, 4)).tolist() == ag.rotary_frequencies(4).tolist() * 2


def test_one_axis_of_positions_may_be_a_stack_of_one():
    """With `sections`, a tensor for each axis, stacked; for one axis also the tensor alone.  (These tensors are on the host, which is all that
    is wrong with them.)"""
    import torch
    from paper_2309_16669_amd import autograd as ag
    q, at, freqs = torch.zeros(3, 6, 4, 64, dtype=torch.bfloat16), torch.arange(6), torch.ones(32)
    for positions, sections in ((at, (32,)), (at[None], (32,)), (at.expand(3, 6), (32,)), (at.expand(1, 3, 6), (32,)), (at, None)):
        with pytest.raises(ValueError, match="must live on the GPU"):
            ag.rotary(q, None, positions, freqs, sections)
    for positions, sections in ((at[None], None), (at.expand(1, 3, 6), None), (at.expand(2, 6), (32,)), (at[None, None], (32,)), (at[:1], (32,))):
        with pytest.raises(ValueError, match="do not fit tokens"):
            ag.rotary(q, None, positions, freqs, sections)


def test_a_gradient_that_rotary_does_not_have_is_refused():
    """A learned spectrum, or learned places between frames, would silently get none."""
    import torch
    from paper_2309_16669_amd import autograd as ag
    q, at, freqs = torch.zeros(6, 4, 64, dtype=torch.bfloat16), torch.arange(6).float(), torch.ones(32)
    for positions, f in ((at, freqs.clone().requires_grad_(True)), (at.clone().requires_grad_(True), freqs),
                         (at, torch.nn.Parameter(freqs) * 2)):
        for k in (None, q[:, :2]):
            with pytest.raises(ValueError, match="no gradient of positions and freqs"):
                ag.rotary(q, k, positions, f)
        with torch.no_grad(), pytest.raises(ValueError, match="must live on the GPU"):
            ag.rotary(q, None, positions, f)
        with pytest.raises(ValueError, match="must live on the GPU"):
            ag.rotary(q, None, positions.detach(), f.detach())


def test_keys_beside_no_query_head_do_not_come_back_as_they_are():
    import torch
    from paper_2309_16669_amd import autograd as ag
    q, k = torch.zeros(6, 0, 64, dtype=torch.bfloat16), torch.ones(6, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="must live on the GPU"):
        ag.rotary(q, k, torch.arange(6), torch.ones(32))


def test_headers_flags_match_the_binding():
    import os
    import re
    text = open(os.path.join(os.path.dirname(av._PKG), "include", "avion_attn.h")).read()
    for name in ("INTERLEAVED", "INVERSE", "POSITIONS_F32", "MEAN", "ONE_GRADIENT"):
        assert int(re.search(rf"#define AVION_FLAG_{name} (\d+)u", text)[1]) == getattr(av, f"FLAG_{name}")
