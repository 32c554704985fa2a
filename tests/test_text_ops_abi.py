"""Token table, RMS normalisation and 8-bit path: what the C entry points and the front end refuse, before anything is
launched.  Runs without a GPU."""
import ctypes

import pytest

import paper_2309_16669_amd as av

P = 0x1000          # aligned, never dereferenced on these paths
f = ctypes.c_float


def _embedding_fwd(tokens=P, table=P, y=P, n=4, V=10, D=64, scale=1.0, flags=0):
    return av.load_library().avion_embedding_fwd(tokens, table, y, n, V, D, f(scale), flags, None)


def _embedding_bwd(tokens=P, dy=P, dtable=P, n=4000, V=10, D=64, scale=1.0, flags=0, ws=P, ws_bytes=1 << 40):
    return av.load_library().avion_embedding_bwd(tokens, dy, dtable, n, V, D, f(scale), flags, ws, ws_bytes, None)


def _rms_fwd(x=P, residual=P, weight=P, y=P, h=P, rstd=P, M=4, D=64, eps=1e-6, flags=0):
    return av.load_library().avion_rmsnorm_fwd(x, residual, weight, y, h, rstd, M, D, f(eps), flags, None)


def _rms_bwd(h=P, weight=P, rstd=P, dy=P, dh=P, dx=P, dr=None, dw=P, M=4, D=64, flags=0, ws=P, ws_bytes=1 << 40):
    return av.load_library().avion_rmsnorm_bwd(h, weight, rstd, dy, dh, dx, dr, dw, M, D, flags, ws, ws_bytes, None)


def _rms_fp8(x=P, residual=P, weight=P, y8=P, scale=P, h=P, M=4, D=64, eps=1e-6, flags=0):
    return av.load_library().avion_rmsnorm_fwd_fp8(x, residual, weight, y8, scale, h, M, D, f(eps), flags, None)


def _quantize(x=P, x8=P, scale=P, M=4, D=64, flags=0):
    return av.load_library().avion_quantize_rows(x, x8, scale, M, D, flags, None)


def _linear(x8=P, xs=P, w8=P, ws=P, bias=None, y=P, M=4, N=64, K=64, flags=0):
    return av.load_library().avion_linear_fp8(x8, xs, w8, ws, bias, y, M, N, K, flags, None)


INF, NAN = float("inf"), float("nan")
CASES = [
    (_embedding_fwd, [(dict(tokens=None), av.EINVAL), (dict(table=None), av.EINVAL), (dict(y=None), av.EINVAL), (dict(n=-1), av.EINVAL),
                      (dict(V=0), av.EINVAL), (dict(D=0), av.EINVAL), (dict(scale=NAN), av.EINVAL), (dict(scale=INF), av.EINVAL),
                      (dict(flags=2), av.EINVAL), (dict(flags=32), av.EINVAL), (dict(D=60), av.EUNSUPPORTED),
                      (dict(D=65536 + 8), av.EUNSUPPORTED), (dict(V=(1 << 28) + 1), av.EUNSUPPORTED),
                      (dict(n=(1 << 28) + 1), av.EUNSUPPORTED), (dict(n=1 << 28, D=264), av.EUNSUPPORTED), (dict(table=P + 8), av.EUNSUPPORTED),
                      (dict(y=P + 2), av.EUNSUPPORTED), (dict(tokens=P + 4), av.EUNSUPPORTED),
                      (dict(tokens=P + 2, flags=av.FLAG_TOKENS_I32), av.EUNSUPPORTED), (dict(n=0, tokens=None, y=None), av.OK)]),
    (_embedding_bwd, [(dict(tokens=None), av.EINVAL), (dict(dy=None), av.EINVAL), (dict(dtable=None), av.EINVAL), (dict(n=-1), av.EINVAL),
                      (dict(scale=INF), av.EINVAL), (dict(flags=4), av.EINVAL), (dict(D=4), av.EUNSUPPORTED),
                      (dict(dy=P + 8), av.EUNSUPPORTED), (dict(dtable=P + 8), av.EUNSUPPORTED), (dict(tokens=P + 1), av.EUNSUPPORTED),
                      (dict(ws=None), av.EWORKSPACE), (dict(ws=P + 16), av.EWORKSPACE), (dict(ws_bytes=4096), av.EWORKSPACE),
                      (dict(n=3, ws_bytes=255), av.EWORKSPACE)]),
    (_rms_fwd, [(dict(x=None), av.EINVAL), (dict(weight=None), av.EINVAL), (dict(y=None), av.EINVAL), (dict(h=None), av.EINVAL),
                (dict(residual=None), av.EINVAL), (dict(residual=None, h=None, flags=av.FLAG_WIDE_F32), av.EINVAL), (dict(M=-1), av.EINVAL),
                (dict(D=0), av.EINVAL), (dict(eps=-1.0), av.EINVAL), (dict(eps=NAN), av.EINVAL), (dict(eps=INF), av.EINVAL),
                (dict(flags=2), av.EINVAL), (dict(flags=16), av.EINVAL), (dict(D=12), av.EUNSUPPORTED), (dict(D=16384 + 8), av.EUNSUPPORTED),
                (dict(x=P + 8), av.EUNSUPPORTED), (dict(rstd=P + 4), av.EUNSUPPORTED), (dict(M=(1 << 40) + 1), av.EUNSUPPORTED),
                (dict(M=0, x=None, y=None), av.OK)]),
    (_rms_bwd, [(dict(h=None), av.EINVAL), (dict(weight=None), av.EINVAL), (dict(rstd=None), av.EINVAL), (dict(dy=None), av.EINVAL),
                (dict(dw=None), av.EINVAL), (dict(dr=P), av.EINVAL), (dict(M=-1), av.EINVAL), (dict(flags=1 << 30), av.EINVAL),
                (dict(D=20), av.EUNSUPPORTED), (dict(dh=P + 8), av.EUNSUPPORTED), (dict(dx=P + 8), av.EUNSUPPORTED),
                (dict(ws=None), av.EWORKSPACE), (dict(ws=P + 128), av.EWORKSPACE), (dict(ws_bytes=255), av.EWORKSPACE)]),
    (_rms_fp8, [(dict(x=None), av.EINVAL), (dict(scale=None), av.EINVAL), (dict(h=None), av.EINVAL), (dict(D=72), av.EUNSUPPORTED),
                (dict(y8=P + 8), av.EUNSUPPORTED), (dict(eps=-1.0), av.EINVAL), (dict(flags=2), av.EINVAL), (dict(M=0), av.OK)]),
    (_quantize, [(dict(x=None), av.EINVAL), (dict(x8=None), av.EINVAL), (dict(scale=None), av.EINVAL), (dict(M=-1), av.EINVAL),
                 (dict(flags=av.FLAG_WIDE_F32), av.EINVAL), (dict(D=72), av.EUNSUPPORTED), (dict(D=1 << 15), av.EUNSUPPORTED),
                 (dict(x=P + 4), av.EUNSUPPORTED), (dict(M=0, x=None), av.OK)]),
    (_linear, [(dict(x8=None), av.EINVAL), (dict(xs=None), av.EINVAL), (dict(w8=None), av.EINVAL), (dict(ws=None), av.EINVAL),
               (dict(y=None), av.EINVAL), (dict(M=-1), av.EINVAL), (dict(N=0), av.EINVAL), (dict(K=0), av.EINVAL), (dict(flags=2), av.EINVAL),
               (dict(N=60), av.EUNSUPPORTED), (dict(K=24), av.EUNSUPPORTED), (dict(K=65536 + 16), av.EUNSUPPORTED),
               (dict(N=(1 << 20) + 8), av.EUNSUPPORTED), (dict(M=1 << 31), av.EUNSUPPORTED), (dict(bias=P + 8), av.EUNSUPPORTED), (dict(x8=P + 8), av.EUNSUPPORTED), (dict(xs=P + 2), av.EUNSUPPORTED),
               (dict(ws=P + 4), av.EUNSUPPORTED),
               (dict(M=0, x8=None, y=None), av.OK)]),
]


@pytest.mark.parametrize("call,kwargs,code", [(c, k, r) for c, cases in CASES for k, r in cases],
                         ids=lambda v: getattr(v, "__name__", None) or str(v))
def test_refused_without_launching(call, kwargs, code):
    assert call(**kwargs) == code


def test_linear_refuses_more_tiles_than_a_launch_holds():
    assert _linear(M=1 << 30, N=128) == av.EUNSUPPORTED


def test_workspace_sizes():
    assert av.embedding_bwd_workspace_bytes(-1, 10, 64) == 0 and av.embedding_bwd_workspace_bytes(10, 10, 12) == 0
    assert av.embedding_bwd_workspace_bytes(0, 10, 64) == 256 and av.embedding_bwd_workspace_bytes(512, 1 << 20, 64) == 256
    a, b = av.embedding_bwd_workspace_bytes(100000, 1000, 64), av.embedding_bwd_workspace_bytes(200000, 1000, 64)
    assert a % 256 == 0 and 100000 * 16 < a < b <= 2 * a + (1 << 20)
    assert av.embedding_bwd_workspace_bytes(1 << 28, 1 << 28, 8) > 1 << 32   # in size_t throughout
    assert av.rmsnorm_bwd_workspace_bytes(5, 12) == 0 and av.rmsnorm_bwd_workspace_bytes(0, 64) == 256
    assert av.rmsnorm_bwd_workspace_bytes(10 ** 6, 768) == av.rmsnorm_bwd_workspace_bytes(10 ** 7, 768)


def test_the_front_end_refuses():
    import torch
    from paper_2309_16669_amd import autograd as ag
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    x, w = torch.zeros(3, 64, dtype=bf), torch.ones(64)
    t, table = torch.zeros(3, dtype=torch.int64), torch.zeros(5, 64, dtype=bf)
    x8, s, w8, ws = torch.zeros(3, 64).to(f8), torch.ones(3), torch.zeros(8, 64).to(f8), torch.ones(8)
    bad = [lambda: ag.embedding(t, table), lambda: ag.embedding(t.short(), table), lambda: ag.embedding(t, table, dtype=torch.float32),
           lambda: ag.embedding(t, table.half(), dtype=bf), lambda: ag.embedding(t, table.double()),
           lambda: ag.rms_norm(x, w), lambda: ag.rms_norm(x.float(), w), lambda: ag.add_rms_norm(x, x[:2], w),
           lambda: ag.add_rms_norm(x, x[0], w), lambda: ag.add_rms_norm(x, x.half(), w), lambda: ag.add_rms_norm_fp8(x, x[:, :8], w),
           lambda: ag.quantize_rows(x.float()), lambda: ag.rms_norm_fp8(x, w), lambda: ag.linear_fp8(x8, s, w8, ws),
           lambda: ag.linear_fp8(x8, s[:2], w8, ws), lambda: ag.linear_fp8(x8, s, w8[:, :16], ws),
           lambda: ag.linear_fp8(x8, s, w8, ws, dtype=torch.float32), lambda: ag.linear_fp8(x8, s, w8[0], ws)]
    for call in bad:   # on the host, or in another format or shape
        with pytest.raises(ValueError):
            call()
    g = w.clone().requires_grad_()
    for call in (lambda: ag.rms_norm_fp8(x, g), lambda: ag.add_rms_norm_fp8(x, x, g),
                 lambda: ag.quantize_rows(x.clone().requires_grad_()), lambda: ag.linear_fp8(x8, s, w8, ws, ws.clone().requires_grad_())):
        with pytest.raises(ValueError, match="no backward"):
            call()


def test_sizes_past_32_bits_are_not_cut():
    # D is an int of the C interface
    with pytest.raises(ValueError, match="32 bits"):
        av._launch(0, av.load_library().avion_quantize_rows, (P, P, P, 1, (1 << 32) + 64, 0), None)
