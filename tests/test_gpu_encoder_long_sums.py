"""GPU test of the parameter gradients that are sums over a whole text, where inputs are mostly positive, as SiLU leaves them: an
error of the same sign at every position, however small, adds up there.

With states that hardly forget, grad_dt_bias is the sum of x . du over the positions (times a sigmoid).  A position's term is off by
some 2^-23 of the terms' size at random, so the sum by 2^-23 of the terms' 2-norm: 1e-6 of it bounds that with room.  An error
of 2e-8 downwards in each would leave 5e-6 over 64 000 positions."""
import numpy as np
import pytest
import torch

from test_gpu_encoder_long_segments import recurrence
from test_gpu_encoder_scan import backward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_errors_do_not_add_up(dtype):
    print("[case] ssm long sums", dtype, flush=True)
    B, T, P, N = 64, 1000, 64, 16
    d, h = make(B, T, 1, P, 1, N, dtype, seed=107, dt_scale=0.1)
    d["xbc"].copy_(torch.nn.functional.silu(d["xbc"].float()).to(dtype))  # x, b and c are views of it
    for k, v in (("dt_bias", np.log(np.expm1(1e-2))), ("rate", -1e-3), ("glast", 0.0)):
        d[k].fill_(float(v))
    for k in ("x", "b", "c", "dt_bias", "rate", "glast"):
        h[k] = d[k].double().cpu().numpy()
    ref, got = recurrence(h), backward(d)
    off = abs(got["grad_dt_bias"].item() - ref["grad_dt_bias"][0]) / np.linalg.norm(ref["grad_dt"])
    print("  off by %.1e of the terms' norm" % off)
    assert off < 1e-6
