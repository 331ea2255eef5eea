"""GPU tests of the embedding's gradient where positions without a token end anywhere in the pieces that its sum is cut into
(16 or 64 sorted positions).  Whole numbers, whose sums are exact."""
import pytest
import torch

from paper_2604_18780_amd import binding as sb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("B,T,valid", [(1, 500, v) for v in (0, 1, 7, 8, 9, 15, 16, 17, 32, 33, 500)] +
                         [(3, 100_000, v) for v in (1, 63, 64, 65, 8191, 90_001)])
@pytest.mark.parametrize("by_length", [True, False])
def test_padding_ends_anywhere(B, T, valid, by_length):
    """The first sequence has `valid` tokens, the others none: by their lengths, or by tokens outside the table."""
    print("[case] embed padding", B, T, valid, by_length, flush=True)
    V, D = 5, 72
    g = torch.Generator(device=DEV).manual_seed(89)
    tokens = torch.randint(0, V, (B, T), generator=g, device=DEV, dtype=torch.int32)
    grad = torch.randint(-8, 9, (B, T, D), generator=g, device=DEV).float()
    ref = torch.zeros(V, D, device=DEV).index_add_(0, tokens[0, :valid].long(), grad[0, :valid])
    lengths = None
    if by_length:
        lengths = torch.zeros(B, dtype=torch.int32, device=DEV)
        lengths[0] = valid
    else:
        tokens[1:], tokens[0, valid:] = V, -1
    grad[1:], grad[0, valid:] = float("nan"), float("nan")
    assert torch.equal(sb.semicrf_embed_bwd(tokens, grad, V, 1.0, lengths), ref)
