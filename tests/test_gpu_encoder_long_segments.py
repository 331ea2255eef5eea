"""GPU tests of the scan and its gradients with segments of 576 and 1024 positions (18 and 32 blocks of the walk that the gradients
of the steps take), states that last for thousands of positions and such that last for tens, against the 64-bit recurrence.

Tolerances (2-norm, relative) as for short segments: 2^-8 for outputs in bfloat16, 1e-5 in float32 and for states and parameter
gradients.  A walk adds up to 64 values in 64 bits, each off by 2^-24 of its terms; what they are off by at its end is
taken back; so positions are off by a few 2^-24 of the pairs that pass them, which a gradient of the steps is about as large as."""
import ctypes

import numpy as np
import pytest
import torch

import encoder_plain as plain
from paper_2604_18780_amd import binding as sb
from test_gpu_encoder_scan import F32_TOL, TOL, backward, far, forward, make

pytestmark = pytest.mark.gpu


def recurrence(h):
    """Outputs, final state and all gradients in 64 bits, one head and one group, every sequence at once."""
    x, b, c, dt = h["x"][:, :, 0], h["b"][:, :, 0], h["c"][:, :, 0], h["dt"][:, :, 0]
    gy, (rate,), (skip,), (bias,) = h["gy"][:, :, 0], h["rate"], h["skip"], h["dt_bias"]
    B, T, _ = x.shape
    live = np.arange(T)[None, :] < np.asarray(h["lengths"])[:, None]
    raw = dt + bias
    delta = np.where(live, plain.softplus(raw), 0.0)
    keep, sg = np.exp(delta * rate), plain.sigmoid(raw)
    state = h["state"][:, 0].copy()
    before, y = np.empty((T,) + state.shape), np.zeros_like(x)
    for t in range(T):
        before[t] = state
        state = keep[:, t, None, None] * state + (delta[:, t, None] * x[:, t])[:, :, None] * b[:, t, None, :]
        y[:, t] = (np.einsum("bpn,bn->bp", state, c[:, t]) + skip * x[:, t]) * live[:, t, None]
    out = dict(y=y[:, :, None], last=state[:, None])
    g = h["glast"][:, 0].copy()
    gx, gb, gc, gdt = np.zeros_like(x), np.zeros_like(b), np.zeros_like(c), np.zeros_like(dt)
    grate = 0.0
    for t in range(T - 1, -1, -1):
        on = live[:, t, None]
        decayed = keep[:, t, None, None] * before[t]
        gyt = gy[:, t] * on
        u = delta[:, t, None] * x[:, t]
        gc[:, t] = np.einsum("bpn,bp->bn", decayed + u[:, :, None] * b[:, t, None, :], gyt)
        g = g + gyt[:, :, None] * c[:, t, None, :]
        du = np.einsum("bpn,bn->bp", g, b[:, t])
        gb[:, t] = np.einsum("bpn,bp->bn", g, u)
        gx[:, t] = (delta[:, t, None] * du + skip * gyt) * on
        dl = np.einsum("bpn,bpn->b", g, decayed) * live[:, t]
        grate += (delta[:, t] * dl).sum()
        gdt[:, t] = ((x[:, t] * du).sum(1) * live[:, t] + rate * dl) * sg[:, t]
        g = keep[:, t, None, None] * g
    out.update(grad_x=gx[:, :, None], grad_b=gb[:, :, None], grad_c=gc[:, :, None], grad_dt=gdt[:, :, None],
               grad_rate=np.array([grate]), grad_skip=np.array([(x * gy * live[:, :, None]).sum()]),
               grad_dt_bias=np.array([gdt.sum()]), grad_state=g[:, None])
    return out


def test_the_recurrence_is_the_plain_one():
    _, h = make(3, 40, 1, 8, 1, 8, torch.float32, [40, 0, 13], seed=101)
    args = [h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")]
    mine, ref = recurrence(h), plain.scan_grad(*args, h["gy"], h["glast"])
    ref["y"], ref["last"], _ = plain.scan(*args)
    for k, r in ref.items():
        assert np.allclose(mine[k], r, rtol=1e-12, atol=1e-12), k


def workspace(B, T, P, N, nseg):
    """Bytes that gradients of one head and one group ask for in `nseg` segments."""
    whole = lambda n: (n + 255) // 256 * 256  # noqa: E731
    states = B * (nseg + 1) * P * N * 4
    return (2 * whole(states) + whole(B * nseg * 4) + 4 * whole(B * T * 4) + whole(B * nseg * 8) + whole(B * nseg * 16)
            + whole(B * (nseg + 1) * ((P * N // 4 + 63) // 64) * 8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("step", [1e-4, 1e-3, 1e-2])
@pytest.mark.parametrize("B,seg", [(200, 576), (400, 1024)])
def test_long_walks(B, seg, step, dtype):
    print("[case] ssm walk", B, seg, step, dtype, flush=True)
    T, P, N = 2100, 8, 8
    n = ctypes.c_size_t(0)
    assert sb.load().semicrf_ssm_workspace_bytes(B, T, 1, P, 1, N, 1, ctypes.byref(n)) == 0
    assert n.value == workspace(B, T, P, N, (T + seg - 1) // seg)
    lengths = np.random.default_rng(7).integers(0, T + 1, B)
    lengths[:B // 2] = T
    d, h = make(B, T, 1, P, 1, N, dtype, lengths, seed=103, garbage=False)
    past = torch.arange(T)[None, :] >= torch.as_tensor(lengths)[:, None]
    for k in ("xbc", "dt", "gy"):
        d[k][past.to(d[k].device)] = float("nan")
    for k, v in (("dt_bias", np.log(np.expm1(step))), ("rate", -1.3)):
        d[k].fill_(float(v))
        h[k] = d[k].double().cpu().numpy()
    ref = recurrence(h)
    y, last = forward(d)
    got = dict(y=y, last=last, **backward(d))
    off = {}
    for k, r in ref.items():
        off[k] = far(got[k], r), (TOL[dtype] if k in ("y", "grad_x", "grad_b", "grad_c", "grad_dt") else F32_TOL)
    print("  " + "  ".join("%s %.1e" % (k, v[0]) for k, v in off.items()))
    for k, (v, limit) in off.items():
        assert v < limit, k
