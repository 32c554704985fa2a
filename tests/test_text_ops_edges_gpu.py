"""GPU tests of the text operators at the ends of their ranges.

Bounds as in test_text_ops_gpu.py: E = 2^-24 for each fp32 operation, u half a step of a result's format."""
import pytest

from oracle import text_ops as ops
from tests.test_text_ops_gpu import E, FP, _rows8_check, f64, randn

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- 8 bits
@pytest.mark.parametrize("h_size,w_size", [(100.0, 2e37), (1e10, 1e30), (1e15, 1e25)])
@pytest.mark.parametrize("M,D", [(5, 64), (9, 256), (3, 768), (600, 768), (2, 4096), (2, 8208)])
def test_rows_in_8_bits_products_past_fp32(h_size, w_size, M, D):
    """h w lies beyond fp32's largest number, y = h rstd w does not; every other row's products are ordinary ones."""
    import torch
    from paper_2309_16669_amd import autograd as ag
    w = w_size * (1 + 0.1 * randn(1, (D,), FP))
    r = h_size * randn(2, (M, D), FP)
    r[1::2] *= 1e-12
    x = torch.zeros((M, D), dtype=torch.bfloat16, device="cuda")
    y, h = ag.add_rms_norm(x, r, w, 1e-20)
    assert torch.equal(h, r) and y.isfinite().all()
    q, s, h = ag.add_rms_norm_fp8(x, r, w, 1e-20)
    assert torch.equal(h, r)
    _rows8_check(ops.rms_fwd(f64(r), f64(w), 1e-20)[0], q, s, (D / 2 + 20) * E)
    if h_size < 1e4:    # the same without a residual, and with ordinary gains on the same rows
        q, s = ag.rms_norm_fp8(r.to(torch.bfloat16), w, 1e-20)
        _rows8_check(ops.rms_fwd(f64(r.to(torch.bfloat16)), f64(w), 1e-20)[0], q, s, (D / 2 + 20) * E)
    q, s, h = ag.add_rms_norm_fp8(x, r, w / w_size, 1e-20)
    _rows8_check(ops.rms_fwd(f64(r), f64(w / w_size), 1e-20)[0], q, s, (D / 2 + 20) * E)
