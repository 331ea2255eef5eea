"""GPU tests of the embedding and of the short convolution (semicrf_embed_*, semicrf_conv_*) and of the single-token step
(semicrf_ssm_step) against the 64-bit forms.

Tolerances (2-norm, relative): an output stored in 2 bytes is rounded once (2^-9 at most for bfloat16, 2^-12 for float16):
2^-8 and 2^-11; float32 outputs are sums of a few products and one sigmoid: 1e-6, table and filter gradients sums of some
thousand terms in 32 bits or more: 2e-6."""
import ctypes

import numpy as np
import pytest
import torch

import encoder_plain as plain
from paper_2604_18780_amd import binding as sb
from test_gpu_encoder_scan import far, make

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TOL = {torch.float32: 1e-6, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def host(t):
    return t.double().cpu().numpy()


# ---- embedding ------------------------------------------------------------------------------------------------------

def text(B, T, V, seed, skew=False, outside=True):
    rng = np.random.default_rng(seed)
    r = rng.random((B, T))
    tokens = ((r ** 6 if skew else r) * V).astype(np.int32)
    if outside:
        tokens[rng.random((B, T)) < 0.1] = -1
        tokens[rng.random((B, T)) < 0.05] = V + 3
    return tokens


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,V,D,lengths,skew", [
    (1, 1, 1, 8, None, False), (1, 1, 300, 512, [0], False), (3, 17, 5, 24, [17, 0, 4], False), (2, 700, 256, 64, None, True),
    (4, 512, 257, 1032, [512, 511, 1, 300], True), (1, 5000, 66000, 40, None, False), (2, 3000, 1, 72, None, False),
    (5, 2000, 7, 136, None, True)])
def test_embedding_and_its_gradient(B, T, V, D, lengths, skew, dtype):
    print("[case] embed", B, T, V, D, dtype, flush=True)
    rng = np.random.default_rng(1)
    tokens = text(B, T, V, 2, skew)
    L = np.full(B, T) if lengths is None else np.asarray(lengths)
    table = torch.from_numpy(rng.standard_normal((V, D))).to(dtype).to(DEV)
    grad = torch.from_numpy(rng.standard_normal((B, T, D))).to(dtype).to(DEV)
    grad[torch.arange(T)[None, :].expand(B, T).to(DEV) >= torch.as_tensor(L, device=DEV)[:, None]] = float("nan")
    tok = torch.from_numpy(tokens).to(DEV)
    lens = None if lengths is None else torch.as_tensor(L, dtype=torch.int32, device=DEV)
    out = sb.semicrf_embed_fwd(tok, table, 1.7, lens)
    assert far(out, plain.embed(tokens, host(table), np.float32(1.7), L)) < TOL[dtype]
    ref = plain.embed_grad(tokens, np.nan_to_num(host(grad)), V, np.float32(1.7), L)
    first = sb.semicrf_embed_bwd(tok, grad, V, 1.7, lens)
    assert far(first, ref) < 2e-6
    assert torch.equal(first, sb.semicrf_embed_bwd(tok, grad, V, 1.7, lens))
    assert not first[torch.from_numpy(~(ref != 0).any(1)).to(DEV)].any()


def test_long_text_of_few_tokens():
    """More than 2^18 positions (longer chunks), a token of a hundred thousand of them, one of none."""
    B, T, V, D = 3, 100001, 6, 16
    tokens = text(B, T, V - 1, 4, skew=True, outside=False)
    g = torch.Generator(device=DEV).manual_seed(5)
    grad = torch.randn(B, T, D, generator=g, device=DEV)
    got = sb.semicrf_embed_bwd(torch.from_numpy(tokens).to(DEV), grad, V)
    h, ref = host(grad).reshape(-1, D), np.zeros((V, D))
    for v in range(V):
        ref[v] = h[tokens.reshape(-1) == v].sum(0)
    assert far(got, ref) < 2e-6 and not got[V - 1].any()


def test_embedding_refusals():
    tok = torch.zeros(2, 8, dtype=torch.int32, device=DEV)
    with pytest.raises(sb.SemiCRFError) as e:
        sb.semicrf_embed_fwd(tok, torch.zeros(4, 12, device=DEV))
    assert e.value.status == -3
    with pytest.raises(ValueError):
        sb.semicrf_embed_fwd(tok.long(), torch.zeros(4, 16, device=DEV))
    with pytest.raises(sb.SemiCRFError) as e:
        sb.semicrf_embed_bwd(tok, torch.zeros(2, 8, 16, device=DEV), 4, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))
    assert e.value.status == -2
    n = ctypes.c_size_t(0)
    assert sb.load().semicrf_embed_bwd_workspace_bytes(0, 8, 4, 16, ctypes.byref(n)) == -1


# ---- convolution ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,C,W,lengths,linear", [
    (1, 1, 8, 4, None, False), (2, 3, 24, 4, [2, 0], False), (2, 33, 136, 3, [33, 32], False), (3, 64, 40, 2, [1, 64, 31], True),
    (1, 700, 328, 4, None, False), (2, 65, 8, 1, None, False), (70, 50, 16, 4, None, False)])
def test_convolution_and_its_gradient(B, T, C, W, lengths, linear, dtype):
    print("[case] conv", B, T, C, W, dtype, flush=True)
    rng = np.random.default_rng(7)
    L = np.full(B, T) if lengths is None else np.asarray(lengths)
    lens = None if lengths is None else torch.as_tensor(L, dtype=torch.int32, device=DEV)
    wide = torch.from_numpy(rng.standard_normal((B, T, C + 16))).to(dtype).to(DEV)
    grad = torch.from_numpy(rng.standard_normal((B, T, C))).to(dtype).to(DEV)
    past = torch.arange(T)[None, :].expand(B, T).to(DEV) >= torch.as_tensor(L, device=DEV)[:, None]
    wide[past], grad[past] = float("nan"), float("nan")
    u = wide[..., 8:8 + C]
    weight = torch.from_numpy(rng.standard_normal((C, W))).float().to(DEV)
    bias = torch.from_numpy(rng.standard_normal(C)).float().to(DEV)
    flags = sb.SEMICRF_CONV_LINEAR if linear else 0
    hu, hg = np.nan_to_num(host(u)), np.nan_to_num(host(grad))
    out = sb.semicrf_conv_fwd(u, weight, bias, lens, flags=flags)
    assert far(out, plain.conv(hu, host(weight), host(bias), L, linear)[0]) < TOL[dtype]
    gu, gw, gb = sb.semicrf_conv_bwd(u, weight, bias, grad, lens, flags=flags)
    ru, rw, rb = plain.conv_grad(hu, host(weight), host(bias), hg, L, linear)
    assert far(gu, ru) < TOL[dtype] and far(gw, rw) < 2e-6 and far(gb, rb) < 2e-6
    assert not out[past].any() and not gu[past].any()


def test_convolution_gradient_matches_differences():
    rng = np.random.default_rng(9)
    u, w, b, g = (rng.standard_normal(s) for s in ((2, 40, 8), (8, 4), (8,), (2, 40, 8)))
    f32 = lambda v: torch.from_numpy(v).float().to(DEV)  # noqa: E731
    got = [host(v) for v in sb.semicrf_conv_bwd(f32(u), f32(w), f32(b), f32(g))]
    u, w, b, g = (v.astype(np.float32).astype(np.float64) for v in (u, w, b, g))
    f = lambda u, w, b: (plain.conv(u, w, b, [40, 40])[0] * g).sum()  # noqa: E731
    for i, v in enumerate((u, w, b)):
        r = rng.standard_normal(v.shape)
        args = lambda e: [x + e * r if k == i else x for k, x in enumerate((u, w, b))]  # noqa: E731
        want = (f(*args(1e-4)) - f(*args(-1e-4))) / 2e-4
        assert abs((got[i] * r).sum() - want) < 1e-5 * np.linalg.norm(got[i]) * np.linalg.norm(r)


@pytest.mark.parametrize("W", [1, 2, 3, 4])
def test_convolution_taken_in_pieces(W):
    """A sequence in pieces of one, two and more tokens, the ring in place or not, one slot without a sequence."""
    B, T, C = 3, 50, 16
    rng = np.random.default_rng(11)
    u = torch.from_numpy(rng.standard_normal((B, T, C))).float().to(DEV)
    weight = torch.from_numpy(rng.standard_normal((C, W))).float().to(DEV)
    whole = sb.semicrf_conv_fwd(u, weight)
    ring = torch.full((B, C, W), 7.0, device=DEV)
    parts, at = [], 0
    for k, n in enumerate((1, 1, 2, 40, 6)):
        seen = torch.tensor([at, -1, at], dtype=torch.int32, device=DEV)
        other = ring if k % 2 else torch.empty_like(ring)
        parts.append(sb.semicrf_conv_fwd(u[:, at:at + n].contiguous(), weight, ring=ring, seen=seen, ring_out=other))
        ring, at = other, at + n
    got = torch.cat(parts, 1)
    assert torch.allclose(got[[0, 2]], whole[[0, 2]], atol=1e-6) and not got[1].any()
    assert (ring[1] == 7.0).all()
    for p in range(T - W, T):
        assert torch.equal(ring[[0, 2], :, p % W], u[[0, 2], p])


def test_convolution_refusals():
    u = torch.zeros(2, 8, 16, device=DEV)
    w = torch.zeros(16, 4, device=DEV)
    with pytest.raises(sb.SemiCRFError) as e:
        sb.semicrf_conv_fwd(u, torch.zeros(16, 5, device=DEV))
    assert e.value.status == -3
    with pytest.raises(sb.SemiCRFError) as e:
        sb.semicrf_conv_fwd(u, w, ring=torch.zeros(2, 16, 4, device=DEV))  # a ring without how much it has seen
    assert e.value.status == -1
    with pytest.raises(ValueError):
        sb.semicrf_conv_fwd(u, w[:8])
    with pytest.raises(ValueError):
        sb.semicrf_conv_bwd(u, w, None, u.half())


# ---- one more token -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,H,P,G,N,W", [(1, 1, 8, 1, 8, 1), (3, 4, 64, 1, 64, 4), (2, 6, 40, 3, 24, 3), (5, 2, 128, 2, 128, 2),
                                         (1, 3, 72, 1, 104, 4)])
def test_step_follows_the_recurrence(B, H, P, G, N, W, dtype):
    """Six tokens from the beginning; y carries one rounding to the type; state and ring (exact copies) stay in step.  State and y
    are sums of a few products in 32 bits: 2e-6."""
    print("[case] step", B, H, P, G, N, W, dtype, flush=True)
    rng = np.random.default_rng(13)
    C = H * P + 2 * G * N
    row = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(dtype).to(DEV)  # noqa: E731
    par = lambda *s: torch.from_numpy(rng.standard_normal(s)).float().to(DEV)  # noqa: E731
    u, dt = row(B, 6, C + 3), row(B, 6, H)
    weight, bias, rate, skip, dt_bias = par(C, W), par(C), -par(H).abs(), par(H), par(H)
    ring, state = torch.full((B, C, W), float("nan"), dtype=dtype, device=DEV), par(B, H, P, N)
    if B > 1:
        ring[1] = 3.0
    seen = np.zeros(B, dtype=np.int32)
    if B > 1:
        seen[1] = -1
    kept = state.clone()
    a, hring = plain.conv(host(u[..., :C]), host(weight), host(bias), np.full(B, 6))
    x = a[..., :H * P].reshape(B, 6, H, P)
    b, c = (v.reshape(B, 6, G, N) for v in np.split(a[..., H * P:], 2, axis=2))
    ry, rlast, _ = plain.scan(x, b, c, host(dt), *(host(v) for v in (rate, skip, dt_bias)), np.full(B, 6), host(state))
    live = [i for i in range(B) if seen[i] >= 0]
    for t in range(6):
        now = torch.from_numpy(np.where(seen < 0, -1, seen + t).astype(np.int32)).to(DEV)
        out = None if t % 2 else (torch.empty(B, H * P, dtype=dtype, device=DEV), torch.empty_like(ring), torch.empty_like(state))
        y = sb.semicrf_ssm_step(u[:, t, :C], weight, bias, dt[:, t], rate, skip, dt_bias, now, ring, state, groups=G, out=out)
        if out is not None:
            _, ring, state = out
        tol = 2e-6 if dtype == torch.float32 else TOL[dtype]
        assert far(y[live], ry[live, t].reshape(len(live), -1)) < tol
    assert far(state[live], rlast[live]) < 2e-6
    for i in live:
        assert np.array_equal(host(ring[i]), hring[i])
    if B > 1:
        assert torch.equal(state[1], kept[1]) and (ring[1] == 3.0).all() and not y[1].any()


def test_prompt_then_tokens():
    """A prompt through convolution and scan, then token by token, against the prompt that holds them too."""
    B, T, H, P, G, N, W = 2, 80, 2, 64, 1, 64, 4
    C = H * P + 2 * G * N
    d, _ = make(B, T, H, P, G, N, torch.float32, seed=21)
    g = torch.Generator(device=DEV).manual_seed(22)
    weight, bias = torch.randn(C, W, generator=g, device=DEV), torch.randn(C, generator=g, device=DEV)

    def prompt(u, dt, ring, state):
        seen = torch.zeros(B, dtype=torch.int32, device=DEV)
        v = sb.semicrf_conv_fwd(u, weight, bias, ring=ring, seen=seen, ring_out=ring)
        x, b, c = v[..., :H * P].unflatten(2, (H, P)), v[..., H * P:-G * N].unflatten(2, (G, N)), v[..., -G * N:].unflatten(2, (G, N))
        return sb.semicrf_ssm_fwd(x, b, c, dt, d["rate"], d["skip"], d["dt_bias"], None, state, state_out=state)[0]

    new = lambda: (torch.zeros(B, C, W, device=DEV), d["state"].clone())  # noqa: E731
    ring, state = new()
    whole = prompt(d["xbc"], d["dt"], ring, state)
    ring2, state2 = new()
    prompt(d["xbc"][:, :75].contiguous(), d["dt"][:, :75].contiguous(), ring2, state2)
    for t in range(75, T):
        seen = torch.full((B,), t, dtype=torch.int32, device=DEV)
        y = sb.semicrf_ssm_step(d["xbc"][:, t], weight, bias, d["dt"][:, t], d["rate"], d["skip"], d["dt_bias"], seen, ring2,
                                state2)
        assert far(y, host(whole[:, t].reshape(B, -1))) < 1e-5
    assert far(state2, host(state)) < 1e-5 and torch.equal(ring, ring2)


def test_step_in_a_graph():
    """The step captured once and replayed: state and ring go on in place, the count of tokens is the caller's tensor."""
    B, H, P, G, N, W = 2, 2, 64, 1, 64, 4
    C = H * P + 2 * G * N
    g = torch.Generator(device=DEV).manual_seed(31)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    weight, bias, rate, skip, dt_bias = r(C, W), r(C), -r(H).abs(), r(H), r(H)
    us, dts, start = r(5, B, C), r(5, B, H), r(B, H, P, N)

    def begin():
        return torch.zeros(B, C, W, device=DEV), start.clone(), torch.zeros(B, dtype=torch.int32, device=DEV)

    ring, state, seen = begin()
    eager = []
    for t in range(5):
        eager.append(sb.semicrf_ssm_step(us[t], weight, bias, dts[t], rate, skip, dt_bias, seen, ring, state).clone())
        seen += 1
    u, dt, y = us[0].clone(), dts[0].clone(), torch.empty(B, H * P, device=DEV)
    ring2, state2, seen2 = begin()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.semicrf_ssm_step(u, weight, bias, dt, rate, skip, dt_bias, seen2, ring2, state2, out=(y, ring2, state2))
        seen2 += 1
    ring3, state3, seen3 = begin()
    ring2.copy_(ring3), state2.copy_(state3), seen2.copy_(seen3)
    for t in range(5):
        u.copy_(us[t]), dt.copy_(dts[t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager[t])
    assert torch.equal(state2, state) and torch.equal(ring2, ring)


def test_step_refusals():
    H, P, N, W = 2, 64, 64, 4
    C = H * P + 2 * N
    z = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
    args = [z(1, C), z(C, W), z(C), z(1, H), z(H), z(H), z(H), torch.zeros(1, dtype=torch.int32, device=DEV), z(1, C, W),
            z(1, H, P, N)]
    sb.semicrf_ssm_step(*args)
    for k, bad in ((0, z(1, C - 1)), (0, z(1, C).half()), (7, z(1)), (8, z(1, C, 3)), (4, z(H + 1))):
        with pytest.raises(ValueError):
            sb.semicrf_ssm_step(*[bad if i == k else v for i, v in enumerate(args)])
    with pytest.raises(ValueError):
        sb.semicrf_ssm_step(*args[:2], None, *args[3:], groups=2)  # the row has no room for two groups
