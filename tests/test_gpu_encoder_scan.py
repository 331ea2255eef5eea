"""GPU tests of the selective state space scan (semicrf_ssm_fwd, semicrf_ssm_bwd) against the 64-bit recurrence.

Tolerances, for the 2-norm of a difference relative to the result's: an output stored in 2 bytes is rounded once (2^-9 at
most for bfloat16, 2^-12 for float16), and everything before that is held to 2^-17 of a term or better, so 2^-8 and 2^-11
bound it with room; float32 inputs keep 2^-24 of a term, sums of a few hundred grow that to some 1e-6, and gradients of the
steps are sums of both signs: 1e-5.  States and parameter gradients are float32 whatever the type; with 2-byte inputs
their terms keep 2^-17 = 7.6e-6, signs at random: 1e-5 of the norm."""
import numpy as np
import pytest
import torch

import encoder_plain as plain
from paper_2604_18780_amd import binding as sb

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TOL = {torch.float32: 1e-5, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F32_TOL = 1e-5
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def far(a, b):
    """2-norm of a - b relative to b's (absolute where b is zero)."""
    a = a.detach().double().cpu().numpy() if torch.is_tensor(a) else np.asarray(a)
    n = np.linalg.norm(b)
    assert np.isfinite(a).all()
    return np.linalg.norm(a - b) / (n if n > 0 else 1.0)


def make(B, T, H, P, G, N, dtype, lengths=None, seed=0, garbage=True, dt_scale=0.5):
    """Inputs as columns of one array, as the convolution leaves them; what lies beyond a sequence's end is not a number."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    lengths = np.full(B, T) if lengths is None else np.asarray(lengths)
    width = H * P + 2 * G * N
    xbc, dt, gy = r(B, T, width), dt_scale * r(B, T, H), r(B, T, H, P)
    start = torch.exp(torch.rand(H, generator=g) * np.log(100.0) + np.log(1e-3))
    p = dict(rate=-(1.0 + 15.0 * torch.rand(H, generator=g)), skip=r(H), dt_bias=start + torch.log(-torch.expm1(-start)))
    state, glast = 0.5 * r(B, H, P, N), 0.5 * r(B, H, P, N)
    past = torch.arange(T)[None, :] >= torch.as_tensor(lengths)[:, None]
    if garbage:
        xbc[past], dt[past], gy[past] = float("nan"), float("nan"), float("inf")
    dev = dict(xbc=xbc.to(dtype).to(DEV), dt=dt.to(dtype).to(DEV), gy=gy.to(dtype).to(DEV), state=state.to(DEV),
               glast=glast.to(DEV), lengths=torch.as_tensor(lengths, dtype=torch.int32, device=DEV),
               **{k: v.to(DEV) for k, v in p.items()})
    dev["x"] = dev["xbc"][..., :H * P].unflatten(2, (H, P))
    dev["b"] = dev["xbc"][..., H * P:H * P + G * N].unflatten(2, (G, N))
    dev["c"] = dev["xbc"][..., H * P + G * N:].unflatten(2, (G, N))
    host = {k: np.nan_to_num(v.double().cpu().numpy(), posinf=0.0) for k, v in dev.items() if k != "lengths"}
    host["lengths"] = lengths
    return dev, host


def forward(d, **kw):
    return sb.semicrf_ssm_fwd(d["x"], d["b"], d["c"], d["dt"], d["rate"], d["skip"], d["dt_bias"], d["lengths"], d["state"],
                              **kw)


def backward(d, **kw):
    return sb.semicrf_ssm_bwd(d["x"], d["b"], d["c"], d["dt"], d["rate"], d["skip"], d["dt_bias"], d["gy"], d["lengths"],
                              d["state"], d["glast"], want_state=True, **kw)


SIZES = [  # B, T, H, P, G, N, lengths
    (1, 1, 1, 64, 1, 64, None),
    (2, 2, 3, 8, 1, 8, [2, 1]),
    (3, 33, 2, 64, 1, 64, [0, 1, 33]),
    (2, 31, 4, 32, 2, 16, None),
    (4, 64, 6, 16, 3, 24, [64, 63, 32, 5]),
    (2, 130, 2, 48, 2, 32, [130, 97]),
    (1, 257, 3, 128, 1, 128, None),
    (2, 300, 2, 72, 1, 104, [300, 128]),
    (3, 700, 5, 64, 5, 40, [700, 0, 513]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward_matches_the_recurrence(size, dtype):
    print("[case] ssm fwd", size, dtype, flush=True)
    *s, lengths = size
    d, h = make(*s, dtype, lengths)
    y, last = forward(d)
    ry, rlast, _ = plain.scan(h["x"], h["b"], h["c"], h["dt"], h["rate"], h["skip"], h["dt_bias"], h["lengths"], h["state"])
    assert far(y, ry) < TOL[dtype]
    assert far(last, rlast) < F32_TOL
    for i, n in enumerate(h["lengths"]):
        assert not y[i, n:].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_gradients_match_the_recurrence(size, dtype):
    print("[case] ssm bwd", size, dtype, flush=True)
    *s, lengths = size
    d, h = make(*s, dtype, lengths)
    got = backward(d)
    ref = plain.scan_grad(h["x"], h["b"], h["c"], h["dt"], h["rate"], h["skip"], h["dt_bias"], h["lengths"], h["state"],
                          h["gy"], h["glast"])
    for k, r in ref.items():
        stored = k in ("grad_x", "grad_b", "grad_c", "grad_dt")
        assert far(got[k], r) < (TOL[dtype] if stored else F32_TOL), k
    for i, n in enumerate(h["lengths"]):
        assert not got["grad_xbc"][i, n:].any() and not got["grad_dt"][i, n:].any()


def test_gradients_match_differences():
    """Along random directions of every input: (f(v + e r) - f(v - e r)) / 2e with f computed by the 64-bit recurrence of
    the float32 inputs, f = <y, gy> + <last, glast>; central differences with e = 1e-4 err by some 1e-7."""
    size = (2, 70, 3, 16, 1, 24)
    d, h = make(*size, torch.float32, [70, 41], seed=3)
    got = backward(d)
    rng = np.random.default_rng(0)
    names = {"x": "grad_x", "b": "grad_b", "c": "grad_c", "dt": "grad_dt", "rate": "grad_rate", "skip": "grad_skip",
             "dt_bias": "grad_dt_bias", "state": "grad_state"}

    def f(v):
        y, last, _ = plain.scan(v["x"], v["b"], v["c"], v["dt"], v["rate"], v["skip"], v["dt_bias"], h["lengths"], v["state"])
        return (y * h["gy"]).sum() + (last * h["glast"]).sum()

    for k, gk in names.items():
        r = rng.standard_normal(h[k].shape)
        e = 1e-4
        want = (f({**h, k: h[k] + e * r}) - f({**h, k: h[k] - e * r})) / (2 * e)
        grad = got[gk].double().cpu().numpy()
        assert abs((grad * r).sum() - want) < 1e-5 * np.linalg.norm(grad) * np.linalg.norm(r), k


@pytest.mark.parametrize("dt_scale,shift", [(0.1, -9.0), (3.0, 3.0)])
def test_slow_and_fast_forgetting(dt_scale, shift):
    """Steps of 1e-4 (nothing forgotten over the sequence) and of several units (nothing kept over two tokens)."""
    d, h = make(2, 600, 2, 64, 1, 64, torch.float32, [600, 333], seed=5, dt_scale=dt_scale)
    d["dt_bias"] += shift
    h["dt_bias"] = d["dt_bias"].double().cpu().numpy()
    y, last = forward(d)
    args = [h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")]
    ry, rlast, _ = plain.scan(*args)
    assert far(y, ry) < 1e-5 and far(last, rlast) < 1e-5
    got, ref = backward(d), plain.scan_grad(*args, h["gy"], h["glast"])
    for k, r in ref.items():
        assert far(got[k], r) < 1e-5, k


def test_a_prompt_taken_in_pieces_and_long_sequences():
    """Pieces of 1, 500 and the rest, state in place, against the whole in one call (which is cut into segments itself)."""
    B, T, H, P, G, N = 1, 5000, 2, 64, 1, 64
    d, _ = make(B, T, H, P, G, N, torch.bfloat16, seed=8)
    y, last = forward(d)
    state = d["state"].clone()
    parts = []
    for a, e in ((0, 1), (1, 501), (501, T)):
        cut = {k: d[k][:, a:e] for k in ("x", "b", "c", "dt")}
        o, _ = sb.semicrf_ssm_fwd(cut["x"], cut["b"], cut["c"], cut["dt"], d["rate"], d["skip"], d["dt_bias"], None, state,
                                  state_out=state)
        parts.append(o)
    assert far(torch.cat(parts, 1), y.double().cpu().numpy()) < 2.0 ** -8
    assert far(state, last.double().cpu().numpy()) < 1e-5


def test_optional_arguments_and_equal_bits():
    d, h = make(2, 200, 2, 64, 1, 64, torch.bfloat16, seed=9)
    zero = np.zeros(2)
    y, none = sb.semicrf_ssm_fwd(d["x"], d["b"], d["c"], d["dt"], d["rate"], want_state=False)
    ry, _, _ = plain.scan(h["x"], h["b"], h["c"], h["dt"], h["rate"], zero, zero, [200, 200], 0 * h["state"])
    assert none is None and far(y, ry) < 2.0 ** -8
    one, two = backward(d), backward(d)
    assert all(torch.equal(one[k], two[k]) for k in one)
    a = sb.semicrf_ssm_bwd(d["x"], d["b"], d["c"], d["dt"], d["rate"], None, None, d["gy"])
    r = plain.scan_grad(h["x"], h["b"], h["c"], h["dt"], h["rate"], zero, zero, [200, 200], 0 * h["state"], h["gy"],
                        0 * h["glast"])
    assert far(a["grad_x"], r["grad_x"]) < 2.0 ** -8 and far(a["grad_rate"], r["grad_rate"]) < 1e-5


def test_other_sequences_keep_their_results():
    """Not-a-numbers in one sequence's valid rows stay in that sequence."""
    d, _ = make(3, 90, 2, 64, 1, 64, torch.bfloat16, seed=10)
    y, last = forward(d)
    d["xbc"][1, 40] = float("nan")
    y2, last2 = forward(d)
    for i in (0, 2):
        assert torch.equal(y[i], y2[i]) and torch.equal(last[i], last2[i])
    assert torch.equal(y[1, :32], y2[1, :32])


def test_on_another_stream():
    d, _ = make(2, 400, 2, 64, 1, 64, torch.bfloat16, seed=11)
    y, last = forward(d)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y2, last2 = forward(d)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(last, last2)


def test_refusals():
    d, _ = make(2, 40, 2, 64, 1, 64, torch.bfloat16, seed=12)
    lib = sb.load()
    import ctypes
    n = ctypes.c_size_t(0)
    size = lambda *a: lib.semicrf_ssm_workspace_bytes(*a, 0, ctypes.byref(n))  # noqa: E731
    assert size(0, 8, 2, 64, 1, 64) == -1 and size(2, 8, 3, 64, 2, 64) == -1
    assert size(2, 8, 2, 60, 1, 64) == -3 and size(2, 8, 2, 64, 1, 136) == -3
    assert lib.semicrf_ssm_workspace_bytes(2, 8, 2, 64, 1, 64, 0, None) == -1
    with pytest.raises(ValueError):  # dt of another type
        sb.semicrf_ssm_fwd(d["x"], d["b"], d["c"], d["dt"].float(), d["rate"])
    with pytest.raises(ValueError):  # heads that do not lie side by side
        sb.semicrf_ssm_fwd(d["x"].transpose(2, 3).contiguous().transpose(2, 3), d["b"], d["c"], d["dt"], d["rate"])
    wide = torch.zeros(2, 40, 2 * 64 + 4, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(sb.SemiCRFError):  # rows that do not begin on 16 bytes
        sb.semicrf_ssm_fwd(wide[..., 4:].unflatten(2, (2, 64)), d["b"], d["c"], d["dt"], d["rate"])
    small = torch.empty(16, dtype=torch.uint8, device=DEV)
    with pytest.raises(sb.SemiCRFError) as e:
        backward(d, workspace=small)
    assert e.value.status == -2
