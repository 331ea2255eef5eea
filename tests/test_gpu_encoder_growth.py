"""GPU tests of rates that do not forget: zero, and above zero, where states grow.

Tolerances as for rates below zero (2-norm, relative): 2^-8 and 2^-11 for outputs in two bytes, 1e-5 in float32 and for states and
parameter gradients.  Terms keep the same 24 bits; of a growing state the latest are the largest, so sums are no longer than those
of a state that forgets.  The step's y and state are sums of a few products in 32 bits: 2e-6 in float32."""
import numpy as np
import pytest
import torch

import encoder_plain as plain
from paper_2604_18780_amd import binding as sb
from test_gpu_encoder_rows import host
from test_gpu_encoder_scan import DEV, F32_TOL, TOL, TYPES, backward, far, forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(2, 40, 3, 16, 1, 24, [40, 9]), (2, 130, 3, 64, 1, 64, [130, 97]), (1, 300, 2, 128, 1, 128, None),
                                  (260, 20, 4, 64, 1, 64, None), (2, 700, 4, 64, 2, 40, [700, 513])])
def test_scan_and_gradients(size, dtype):
    """Heads between a rate of -1 and one that grows a hundredfold over the sequence; steps are up to some 0.15."""
    print("[case] ssm growth", size, dtype, flush=True)
    *s, lengths = size
    d, h = make(*s, dtype, lengths, seed=61)
    rates = np.linspace(-1.0, 60.0 / s[1], s[2])
    rates[0 if s[2] < 3 else 1] = 0.0
    d["rate"] = torch.from_numpy(rates).float().to(DEV)
    h["rate"] = host(d["rate"])
    args = [h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")]
    y, last = forward(d)
    ry, rlast, _ = plain.scan(*args)
    assert far(y, ry) < TOL[dtype] and far(last, rlast) < F32_TOL
    got, ref = backward(d), plain.scan_grad(*args, h["gy"], h["glast"])
    for k, r in ref.items():
        stored = k in ("grad_x", "grad_b", "grad_c", "grad_dt")
        assert far(got[k], r) < (TOL[dtype] if stored else F32_TOL), k


def test_large_steps_within_sixteen_positions():
    """delta of 0.3 and a rate of 1: e^4.5 over sixteen positions, where a key's weight for a query is largest."""
    d, h = make(1, 30, 2, 64, 1, 64, torch.float32, seed=67, dt_scale=0.0)
    for k, v in (("rate", torch.tensor([1.0, -1.0])), ("dt_bias", torch.full((2,), float(np.log(np.expm1(0.3)))))):
        d[k] = v.float().to(DEV)
        h[k] = host(d[k])
    args = [h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")]
    y, last = forward(d)
    ry, rlast, _ = plain.scan(*args)
    assert far(y, ry) < 1e-5 and far(last, rlast) < 1e-5
    got, ref = backward(d), plain.scan_grad(*args, h["gy"], h["glast"])
    for k, r in ref.items():
        assert far(got[k], r) < 1e-5, k


def test_scan_and_single_tokens_agree():
    B, T, H, P, N, W = 2, 24, 3, 32, 32, 2
    C = H * P + 2 * N
    rng = np.random.default_rng(71)
    f32 = lambda *s: torch.from_numpy(rng.standard_normal(s)).float().to(DEV)  # noqa: E731
    u, dt, weight, bias, skip, dt_bias = f32(B, T, C), f32(B, T, H), f32(C, W), f32(C), f32(H), f32(H) - 2.0
    rate = torch.tensor([-1.0, 0.0, 0.7], device=DEV)
    v = sb.semicrf_conv_fwd(u, weight, bias)
    y, last = sb.semicrf_ssm_fwd(v[..., :H * P].unflatten(2, (H, P)), v[..., H * P:H * P + N].unflatten(2, (1, N)),
                                 v[..., H * P + N:].unflatten(2, (1, N)), dt, rate, skip, dt_bias)
    ring, state = torch.zeros(B, C, W, device=DEV), torch.zeros(B, H, P, N, device=DEV)
    for t in range(T):
        seen = torch.full((B,), t, dtype=torch.int32, device=DEV)
        one = sb.semicrf_ssm_step(u[:, t], weight, bias, dt[:, t], rate, skip, dt_bias, seen, ring, state)
        assert far(one, host(y[:, t].reshape(B, -1))) < 1e-5
    assert far(state, host(last)) < 1e-5
