"""GPU test of the workspaces that a caller may hand to the encoder operators: those that are not device memory, or have gaps, are
refused before anything is launched, and one of another type counts in bytes."""
import pytest
import torch

from paper_2604_18780_amd import binding as sb
from test_gpu_encoder_scan import DEV, backward, forward, make

pytestmark = pytest.mark.gpu


def test_workspaces_are_checked():
    d, _ = make(2, 900, 2, 16, 1, 16, torch.float32, seed=97)
    u, weight = d["xbc"], torch.randn(d["xbc"].shape[2], 3, device=DEV)
    tokens = torch.zeros(2, 900, dtype=torch.int32, device=DEV)
    calls = {
        "scan": lambda w: forward(d, workspace=w), "scan gradients": lambda w: backward(d, workspace=w),
        "convolution gradients": lambda w: sb.semicrf_conv_bwd(u, weight, None, u, workspace=w),
        "embedding gradient": lambda w: sb.semicrf_embed_bwd(tokens, u, 4, workspace=w)}
    big = 64 << 20
    for name, call in calls.items():
        for bad in (torch.empty(big, dtype=torch.uint8), torch.empty(2 * big, dtype=torch.uint8, device=DEV)[::2]):
            with pytest.raises(ValueError):
                call(bad)
        print("[case] workspace", name, flush=True)
        call(torch.empty(big // 8, dtype=torch.float64, device=DEV))
        with pytest.raises(sb.SemiCRFError) as e:
            call(torch.empty(1, dtype=torch.float64, device=DEV))
        assert e.value.status == -2, name
