"""GPU tests of values that are not finite in valid rows of dt: results that depend on them are not finite either, and other
sequences keep their bits."""
import pytest
import torch

from paper_2604_18780_amd import binding as sb
from test_gpu_encoder_scan import DEV, TYPES, backward, forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 40, 600])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_steps_that_are_no_numbers_show(value, T, dtype):
    d, _ = make(2, T, 2, 64, 1, 64, dtype, [T, T], seed=79)
    y, last = forward(d)
    g = backward(d)
    at = T // 2
    d["dt"][0, at, 1] = value
    y2, last2 = forward(d)
    g2 = backward(d)
    assert not y2[0, at, 1].isfinite().any() and not last2[0, 1].isfinite().any()
    assert not g2["grad_dt"][0, at, 1].isfinite() and not g2["grad_rate"][1].isfinite()
    assert torch.equal(y[1], y2[1]) and torch.equal(last[1], last2[1])
    for k in ("grad_xbc", "grad_dt", "grad_state"):
        assert torch.equal(g[k][1], g2[k][1]), k


@pytest.mark.parametrize("dtype", TYPES)
def test_a_step_of_one_token(dtype):
    B, H, P, N, W = 2, 2, 32, 24, 3
    C = H * P + 2 * N
    g = torch.Generator(device=DEV).manual_seed(83)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    u, dt, weight, rate, state = r(B, C).to(dtype), r(B, H).to(dtype), r(C, W), -r(H).abs(), r(B, H, P, N)
    dt[0, 1] = float("nan")
    y = sb.semicrf_ssm_step(u, weight, None, dt, rate, None, None, torch.zeros(B, dtype=torch.int32, device=DEV),
                            torch.zeros(B, C, W, dtype=dtype, device=DEV), state)
    assert y[0, P:].isnan().all() and state[0, 1].isnan().all()
    assert y[0, :P].isfinite().all() and y[1].isfinite().all() and state[0, 0].isfinite().all() and state[1].isfinite().all()
