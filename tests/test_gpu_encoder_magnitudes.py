"""GPU tests of the scan's gradients at magnitudes whose squares float32 does not hold, while every result fits.

Gradients are linear in those of the outputs: multiplied by a power of two, they are the same bits times that power, so
long as nothing overflows or falls below the smallest normal number.  Tolerance against the 64-bit recurrence as at ordinary
magnitudes (1e-5 of the norm in float32, 2^-8 for outputs in bfloat16)."""
import pytest
import torch

import encoder_plain as plain
from test_gpu_encoder_scan import F32_TOL, TOL, backward, far, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [(2, 70, 2, 16, 1, 24, [70, 33]), (1, 600, 2, 64, 1, 64, None), (260, 5, 4, 64, 1, 64, None)])
def test_large_gradients(size, dtype):
    """2^70, about 1e21: pairs of positions reach 1e23, their squares 1e46."""
    print("[case] ssm magnitudes", size, dtype, flush=True)
    *s, lengths = size
    d, h = make(*s, dtype, lengths, seed=73)
    small = backward(d)
    for k in ("gy", "glast"):
        d[k], h[k] = d[k] * 2.0 ** 70, h[k] * 2.0 ** 70
    got = backward(d)
    ref = plain.scan_grad(*[h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")], h["gy"], h["glast"])
    for k, r in ref.items():
        stored = k in ("grad_x", "grad_b", "grad_c", "grad_dt")
        assert far(got[k], r) < (TOL[dtype] if stored else F32_TOL), k
        assert far(got[k].double() / 2.0 ** 70, small[k].double().cpu().numpy()) < 1e-6, k
