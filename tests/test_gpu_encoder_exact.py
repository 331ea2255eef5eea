"""GPU tests of what the scan holds before it rounds an output to two bytes: 24 bits of every term, whatever the type.

An output v is compared with the 64-bit recurrence r: |v - r| is at most half a unit of the type (r rounded), and what v was
off by before it was rounded.  That is held against A, the same output of the inputs' magnitudes, which is the sum of its
terms' magnitudes.  A term is a product of factors that are right to 2^-23 each (parts of 24 bits, two powers of two, two or three
products), 2^-22 at random, and the sums of some hundred of them add as much again: 2^-20 of A bounds it.  Factors of 16 bits
would leave up to 2^-17 of a term."""
import numpy as np
import pytest
import torch

import encoder_plain as plain
from test_gpu_encoder_scan import backward, forward, make

pytestmark = pytest.mark.gpu

BITS = {torch.bfloat16: 8, torch.float16: 11}


def half_unit(r, dtype):
    """Half a unit in the last place of r rounded to the type (of its subnormals at least, for float16)."""
    e = np.floor(np.log2(np.maximum(np.abs(r), 1e-300)))
    e = np.maximum(e, -14) if dtype == torch.float16 else e
    return 0.5 * 2.0 ** (e + 1 - BITS[dtype])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [(2, 300, 4, 64, 1, 64), (260, 6, 4, 64, 1, 64), (1, 400, 2, 128, 1, 128), (2, 257, 4, 32, 2, 128),
                                  (2, 200, 2, 128, 1, 32)])
def test_outputs_are_rounded_once(size, dtype):
    print("[case] ssm rounding", size, dtype, flush=True)
    d, h = make(*size, dtype, seed=53)
    names = ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")
    args = [h[k] for k in names]
    sizes = [h[k] if k in ("dt", "rate", "dt_bias", "lengths") else np.abs(h[k]) for k in names]
    got = dict(y=forward(d)[0], **backward(d))
    ref = dict(y=plain.scan(*args)[0], **plain.scan_grad(*args, h["gy"], h["glast"]))
    most = dict(y=plain.scan(*sizes)[0], **plain.scan_grad(*sizes, np.abs(h["gy"]), np.abs(h["glast"])))
    for k in ("y", "grad_x", "grad_b", "grad_c"):
        v = got[k].double().cpu().numpy()
        over = (np.abs(v - ref[k]) - half_unit(ref[k], dtype)) / most[k]
        flips = (over > 0).mean()
        print("  %s: off by up to 2^%.1f of its terms, %.1e rounded to the other side" % (k, np.log2(max(over.max(), 2.0 ** -40)), flips))
        assert over.max() < 2.0 ** -20, k
