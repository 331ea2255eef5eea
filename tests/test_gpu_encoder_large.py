"""GPU tests of the encoder operators at the sizes from which they take their other forms (several heads to a workgroup, wide
step workgroups, longer runs of the convolution, several segments), with workspaces and outputs that hold not-a-numbers
before the call, and with arrays of more than 2^31 elements.

Tolerances as in the tests of small sizes: 2^-8 and 2^-11 for outputs in two bytes, 1e-5 for the scan in float32 and for its
states and parameter gradients, 1e-6 and 2e-6 for the convolution and the step."""
import ctypes

import numpy as np
import pytest
import torch

import encoder_plain as plain
from paper_2604_18780_amd import binding as sb
from test_gpu_encoder_rows import host
from test_gpu_encoder_scan import F32_TOL, TOL, TYPES, backward, far, forward, make

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def spoilt(entry, *sizes):
    """A workspace of the size that `entry` names, every word of it not a number."""
    n = ctypes.c_size_t(0)
    assert getattr(sb.load(), entry)(*sizes, ctypes.byref(n)) == 0
    return torch.full((max(n.value, 256),), 0xff, dtype=torch.uint8, device=DEV)


HEADS = [  # B, T, H, P, G, N: enough sequences for two heads to a workgroup, the last of an odd number alone
    (260, 3, 4, 16, 1, 24, None),
    (175, 5, 5, 64, 1, 64, None),
    (64, 257, 6, 16, 2, 24, "ragged"),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", HEADS)
def test_gradients_of_several_heads_to_a_workgroup(size, dtype):
    print("[case] ssm bwd heads", size, dtype, flush=True)
    *s, ragged = size
    lengths = np.random.default_rng(4).integers(0, s[1] + 1, s[0]) if ragged else None
    d, h = make(*s, dtype, lengths, seed=17)
    got = backward(d)
    args = [h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")]
    ref = plain.scan_grad(*args, h["gy"], h["glast"])
    for k, r in ref.items():
        stored = k in ("grad_x", "grad_b", "grad_c", "grad_dt")
        assert far(got[k], r) < (TOL[dtype] if stored else F32_TOL), k
    again = backward(d)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,N", [(32, 16), (64, 64), (128, 40)])
def test_several_segments(P, N, dtype):
    """A few thousand positions of few heads: segments of their own, forwards and backwards, for each width."""
    print("[case] ssm segments", P, N, dtype, flush=True)
    d, h = make(2, 1500, 2, P, 1, N, dtype, [1500, 1030], seed=23)
    args = [h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")]
    y, last = forward(d)
    ry, rlast, _ = plain.scan(*args)
    assert far(y, ry) < TOL[dtype] and far(last, rlast) < F32_TOL
    got, ref = backward(d), plain.scan_grad(*args, h["gy"], h["glast"])
    for k, r in ref.items():
        stored = k in ("grad_x", "grad_b", "grad_c", "grad_dt")
        assert far(got[k], r) < (TOL[dtype] if stored else F32_TOL), k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P", [16, 40, 128])
@pytest.mark.parametrize("N", [24, 64, 120])
def test_every_pair_of_widths(P, N, dtype):
    """Narrow heads with wide states and the reverse, each width padded by itself; once with two heads to a workgroup."""
    for B, T, H, lengths in ((2, 70, 3, [70, 45]), (260, 5, 4, None)):
        print("[case] ssm widths", B, P, N, dtype, flush=True)
        d, h = make(B, T, H, P, 1, N, dtype, lengths, seed=47)
        args = [h[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias", "lengths", "state")]
        y, last = forward(d)
        ry, rlast, _ = plain.scan(*args)
        assert far(y, ry) < TOL[dtype] and far(last, rlast) < F32_TOL
        got, ref = backward(d), plain.scan_grad(*args, h["gy"], h["glast"])
        for k, r in ref.items():
            stored = k in ("grad_x", "grad_b", "grad_c", "grad_dt")
            assert far(got[k], r) < (TOL[dtype] if stored else F32_TOL), k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,H,P,G,N,W", [(300, 4, 72, 2, 40, 4), (520, 2, 64, 1, 128, 3)])
def test_step_of_many_streams(B, H, P, G, N, W, dtype):
    print("[case] step", B, H, P, G, N, W, dtype, flush=True)
    rng = np.random.default_rng(29)
    C = H * P + 2 * G * N
    row = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(dtype).to(DEV)  # noqa: E731
    par = lambda *s: torch.from_numpy(rng.standard_normal(s)).float().to(DEV)  # noqa: E731
    u, dt, weight, bias, rate, skip, dt_bias = row(B, 2, C), row(B, 2, H), par(C, W), par(C), -par(H).abs(), par(H), par(H)
    ring, state = torch.full((B, C, W), float("nan"), dtype=dtype, device=DEV), par(B, H, P, N)
    a, _ = plain.conv(host(u), host(weight), host(bias), np.full(B, 2))
    b, c = (v.reshape(B, 2, G, N) for v in np.split(a[..., H * P:], 2, axis=2))
    ry, rlast, _ = plain.scan(a[..., :H * P].reshape(B, 2, H, P), b, c, host(dt), *(host(v) for v in (rate, skip, dt_bias)),
                              np.full(B, 2), host(state))
    idle = torch.arange(B, device=DEV) % 7 == 3
    kept = state.clone()
    for t in range(2):
        seen = torch.where(idle, -1, t).int()
        y = sb.semicrf_ssm_step(u[:, t], weight, bias, dt[:, t], rate, skip, dt_bias, seen, ring, state, groups=G)
        assert not y[idle].any()
        assert far(y[~idle], ry[:, t].reshape(B, -1)[(~idle).cpu().numpy()]) < (2e-6 if dtype == torch.float32 else TOL[dtype])
    assert far(state[~idle], rlast[(~idle).cpu().numpy()]) < 2e-6 and torch.equal(state[idle], kept[idle])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,C,W,ragged", [(3, 3001, 1024, 4, True), (2, 9001, 2056, 3, False), (200, 65, 1024, 2, True)])
def test_convolution_in_longer_runs(B, T, C, W, ragged, dtype):
    """Runs of 16 and 32 positions, and more of them than workgroups; each channel by itself, so some columns stand for all."""
    print("[case] conv runs", B, T, C, W, dtype, flush=True)
    g = torch.Generator(device=DEV).manual_seed(31)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    L = np.random.default_rng(5).integers(1, T + 1, B) if ragged else np.full(B, T)
    lens = torch.as_tensor(L, dtype=torch.int32, device=DEV)
    u, gy, weight, bias = r(B, T, C).to(dtype), r(B, T, C).to(dtype), r(C, W), r(C)
    past = torch.arange(T, device=DEV)[None, :] >= lens[:, None]
    u[past], gy[past] = float("nan"), float("nan")
    out = sb.semicrf_conv_fwd(u, weight, bias, lens)
    gu, gw, gb = sb.semicrf_conv_bwd(u, weight, bias, gy, lens)
    assert not out[past].any() and not gu[past].any()
    pick = [0, 7, 8, C // 2 + 3, C - 1]
    hu, hg = (np.nan_to_num(host(v[..., pick])) for v in (u, gy))
    tol = 1e-6 if dtype == torch.float32 else TOL[dtype]
    assert far(out[..., pick], plain.conv(hu, host(weight[pick]), host(bias[pick]), L)[0]) < tol
    ru, rw, rb = plain.conv_grad(hu, host(weight[pick]), host(bias[pick]), hg, L)
    assert far(gu[..., pick], ru) < tol and far(gw[pick], rw) < 2e-6 and far(gb[pick], rb) < 2e-6


@pytest.mark.parametrize("n,V,D", [(1024, 1000, 8), (1025, 255, 8), (4096, 256, 16), (4097, 70000, 8), (4000, 1 << 21, 8),
                                   (33000, 300, 8), (140_000, 66_000, 8)])
def test_embedding_gradient_by_every_sort(n, V, D):
    """One workgroup, few tiles, many tiles and long ones, one to three passes; whole numbers, whose sums are exact."""
    print("[case] embed sort", n, V, D, flush=True)
    g = torch.Generator(device=DEV).manual_seed(43)
    tokens = (torch.rand(1, n, generator=g, device=DEV) ** 3 * V * 1.02).int()
    tokens[0, ::13] = -5
    grad = torch.randint(-8, 9, (1, n, D), generator=g, device=DEV).float()
    valid = ((tokens >= 0) & (tokens < V))[0]
    ref = torch.zeros(V, D, dtype=torch.float64, device=DEV).index_add_(0, tokens[0][valid].long(), grad[0][valid].double())
    assert torch.equal(sb.semicrf_embed_bwd(tokens, grad, V).double(), ref)


def test_nothing_is_read_before_it_is_written():
    """Workspaces and outputs full of not-a-numbers: the same bits as with fresh ones."""
    d, _ = make(3, 900, 4, 64, 2, 40, torch.bfloat16, [900, 0, 513], seed=37)
    args = [d[k] for k in ("x", "b", "c", "dt", "rate", "skip", "dt_bias")]
    y, last = forward(d)
    y2, last2 = forward(d, workspace=spoilt("semicrf_ssm_workspace_bytes", 3, 900, 4, 64, 2, 40, 0),
                        out=torch.full_like(y, float("nan")), state_out=torch.full_like(last, float("nan")))
    assert torch.equal(y, y2) and torch.equal(last, last2)
    got = backward(d)
    again = sb.semicrf_ssm_bwd(*args, d["gy"], d["lengths"], d["state"], d["glast"], want_state=True,
                               workspace=spoilt("semicrf_ssm_workspace_bytes", 3, 900, 4, 64, 2, 40, 1))
    assert all(torch.equal(got[k], again[k]) for k in got)
    tokens = torch.randint(-1, 50, (3, 900), device=DEV, dtype=torch.int32)
    grad = torch.randn(3, 900, 72, device=DEV)
    table = sb.semicrf_embed_bwd(tokens, grad, 60, 0.5, d["lengths"])
    table2 = sb.semicrf_embed_bwd(tokens, grad, 60, 0.5, d["lengths"], workspace=spoilt("semicrf_embed_bwd_workspace_bytes", 3, 900, 60, 72),
                                  grad_table=torch.full((60, 72), float("nan"), device=DEV))
    assert torch.equal(table, table2)
    u, weight = d["xbc"].nan_to_num(), torch.randn(d["xbc"].shape[2], 4, device=DEV)
    one = sb.semicrf_conv_bwd(u, weight, None, u)
    two = sb.semicrf_conv_bwd(u, weight, None, u, workspace=spoilt("semicrf_conv_bwd_workspace_bytes", 3, 900, u.shape[2], 4))
    assert all(torch.equal(a, b) for a, b in zip(one[:2], two[:2]))


def test_rows_beyond_32_bit_offsets():
    """600 000 positions of 4096 columns: 2.46e9 elements.  The last positions against the same computed from a piece."""
    T, D, back = 600_000, 4096, 700
    g = torch.Generator(device=DEV).manual_seed(41)
    tokens = torch.randint(0, 50, (1, T), generator=g, device=DEV, dtype=torch.int32)
    table = torch.randn(50, D, generator=g, device=DEV).bfloat16()
    u = sb.semicrf_embed_fwd(tokens, table)
    assert torch.equal(u[:, -back:], table[tokens[:, -back:].long()])
    print("[case] embed gradient", flush=True)
    grad = sb.semicrf_embed_bwd(tokens, u, 50)
    count = torch.bincount(tokens[0].long(), minlength=50).double()
    assert far(grad, host(table) * count.cpu().numpy()[:, None]) < 2e-6
    print("[case] convolution", flush=True)
    weight, bias = torch.randn(D, 4, generator=g, device=DEV), torch.randn(D, generator=g, device=DEV)
    v = sb.semicrf_conv_fwd(u, weight, bias)
    piece = u[:, -back - 3:].contiguous()
    assert torch.equal(sb.semicrf_conv_fwd(piece, weight, bias)[:, 3:], v[:, -back:])
    gu, _, _ = sb.semicrf_conv_bwd(u, weight, bias, v)
    gu2, _, _ = sb.semicrf_conv_bwd(piece, weight, bias, v[:, -back - 3:].contiguous())
    assert torch.equal(gu2[:, 3:], gu[:, -back:])
    del gu, gu2
    print("[case] scan", flush=True)
    H, P, N = 30, 128, 128
    x, b, c = v[..., :H * P].unflatten(2, (H, P)), v[..., H * P:H * P + N].unflatten(2, (1, N)), v[..., -N:].unflatten(2, (1, N))
    dt = torch.randn(1, T, H, generator=g, device=DEV).bfloat16()
    rate = -torch.rand(H, generator=g, device=DEV) - 0.5
    y, last = sb.semicrf_ssm_fwd(x, b, c, dt, rate)
    # what is kept over a few hundred steps of softplus(dt) ~ 0.8 is nothing
    cut = lambda t: t[:, -back - 300:]  # noqa: E731
    y2, last2 = sb.semicrf_ssm_fwd(cut(x), cut(b), cut(c), cut(dt), rate)
    assert far(y[:, -back:], host(y2[:, 300:])) < 2.0 ** -8 and far(last, host(last2)) < F32_TOL
    del u, y
    print("[case] scan gradient", flush=True)
    one = sb.semicrf_ssm_bwd(x, b, c, dt, rate, None, None, x)
    two = sb.semicrf_ssm_bwd(cut(x), cut(b), cut(c), cut(dt), rate, None, None, cut(x))
    for k in ("grad_x", "grad_b", "grad_c", "grad_dt"):
        assert far(one[k][:, -back:], host(two[k][:, 300:])) < 2.0 ** -8, k
