"""GPU test of the parameters that a stream of single tokens steps with: laid out when it is made, not for every token.

A stream and the whole text differ by the order of sums in float32 (1e-4 of the largest emission); in bfloat16 the whole text is
rounded to 2^-9 after each of five operators and the stream after four, of terms that may cancel: a tenth."""
import pytest
import torch

from paper_2604_18780_amd import encoder

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_parameters_are_those_of_the_last_refresh(dtype):
    enc = encoder.Encoder(11, 3, width=16, heads=4, channels=8, groups=2, states=8, dtype=dtype, device=DEV, seed=5)
    tokens = torch.randint(0, 11, (2, 12), device=DEV, dtype=torch.int32)
    one, two = encoder.Stream(enc, 2), encoder.Stream(enc, 2)
    for t in range(4):
        assert torch.equal(one.step(tokens[:, t].contiguous()), two.step(tokens[:, t].contiguous()))
    kept = {k: v.clone() for k, v in enc.params.items()}
    expected = [two.step(tokens[:, t].contiguous()) for t in range(4, 8)]
    for v in enc.params.values():
        v.mul_(1.25)
    for t in range(4, 8):
        assert torch.equal(one.step(tokens[:, t].contiguous()), expected[t - 4])
    one.refresh()
    at = tokens[:, 8].contiguous()
    assert not torch.equal(one.step(at), two.step(at))
    for k, v in kept.items():
        enc.params[k].copy_(v)
    third, whole = encoder.Stream(enc, 2), enc.emissions(tokens)[0]
    for t in range(12):
        e = third.step(tokens[:, t].contiguous())
    assert (e - whole[:, 11]).abs().max() < (1e-4 if dtype == torch.float32 else 0.1) * whole.abs().max()
