"""The encoder operators of this library as a user calls them, their plain forms, and the sizes they are used at.

A case is one pass through an operator on a batch of B sequences of up to T tokens:

  op "embed"  mode "score": token embedding with scaling; "train": its gradient with respect to the table as well
  op "conv"   mode "score": short causal convolution with SiLU; "train": with its gradients
  op "scan"   mode "score": selective state space scan from a given state, output and final state; "train": output and
              every gradient
  op "step"   convolution and scan for one more token of each of B streams

Other fields: "type", the storage type of activations; V, D (table); C, W (channels and width of the convolution);
H, P, G, N (heads, channels per head, groups that share B_t and C_t, state size); "ragged", whether lengths are spread
over [T/2, T] with one empty sequence; "skew", whether few tokens make up most of the text.  Batches and lengths are those of
``synth.CONFIGS`` and odd ones around them; widths are those of small encoders in front of a segment model.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
SCAN_WORK = 400_000 * 8 * 64 * 64        # tokens * heads * channels * states of the largest listed scans
TRAIN_TOKENS = 400_000 * 512             # tokens * channels of the largest listed training passes
STEP_WORK = 192 * 16 * 64 * 128
CHUNK = 64                               # positions a plain scan takes at once


def _case(name, op, B, T, mode="score", type="bfloat16", ragged=False, **sizes):
    return dict(name=name, op=op, mode=mode, type=type, B=B, T=T, ragged=ragged, **sizes)


def listed():
    return [
        # one stream annotated as it arrives: nothing but latency
        _case("step_one_stream", "step", 1, 1, H=8, P=64, G=1, N=64, W=4),
        # a server's slots, some of them idle, on a wider encoder
        _case("step_many_streams", "step", 192, 1, ragged=True, H=16, P=64, G=1, N=128, W=4),
        # validation on sentences of up to 256 tokens
        _case("embed_score_sentences", "embed", 64, 256, type="float32", ragged=True, V=5003, D=256, skew=True),
        # training on sentences with a word-piece table: the gradient of a large table from few tokens
        _case("embed_train_sentences", "embed", 64, 256, mode="train", ragged=True, V=32000, D=512, skew=True),
        # training on a genome in six-letter words: many tokens, a table that fits a cache
        _case("embed_train_genome", "embed", 4, 100_000, mode="train", V=4101, D=512, skew=False),
        # training on sentences, float32 and a width that is no power of two
        _case("conv_train_sentences", "conv", 64, 251, mode="train", type="float32", ragged=True, C=328, W=4),
        # training on a genome: x, B and C of the scan below in one call
        _case("conv_train_genome", "conv", 4, 100_000, mode="train", C=640, W=4),
        # a prompt of speech frames, half precision, two groups, before it is continued frame by frame
        _case("scan_score_speech", "scan", 32, 2000, type="float16", ragged=True, H=12, P=64, G=2, N=128),
        # training on sentences in float32, small heads, an odd length
        _case("scan_train_sentences", "scan", 64, 251, mode="train", type="float32", ragged=True, H=6, P=32, G=1, N=32),
        # training on speech
        _case("scan_train_speech", "scan", 32, 1999, mode="train", ragged=True, H=8, P=64, G=1, N=64),
        # training on a genome: the longest training step
        _case("scan_train_genome", "scan", 4, 100_000, mode="train", H=8, P=64, G=1, N=64),
        # one chromosome-sized piece in one call
        _case("scan_score_chromosome", "scan", 1, 400_000, H=8, P=64, G=1, N=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    op = rng.choice(("step", "embed", "embed", "conv", "scan", "scan", "scan"))
    mode = rng.choice(("score", "train", "train"))
    kind = rng.choice(("bfloat16", "bfloat16", "float16", "float32"))
    if op == "embed":
        D = 8 * _log_int(rng, 8, 128)
        # a pass writes the whole table's gradient: the table costs like as many tokens
        V = _log_int(rng, 5, min(100_000, TRAIN_TOKENS // (4 * D)))
        tokens = TRAIN_TOKENS // (2 * D) - V
        B = _log_int(rng, 1, 64)
        T = _log_int(rng, 1, min(100_000, tokens // B))
        return _case(None, op, B, T, mode, kind, B > 1 and rng.random() < 0.6, V=V, D=D, skew=rng.random() < 0.5)
    if op == "conv":
        C = 8 * _log_int(rng, 4, 256)
        B = _log_int(rng, 1, 64)
        T = _log_int(rng, 1, min(100_000, TRAIN_TOKENS // (2 * C * B)))
        return _case(None, op, B, T, mode, kind, B > 1 and rng.random() < 0.6, C=C, W=rng.choice((2, 3, 4, 4)))
    G = rng.choice((1, 1, 1, 2, 3))
    H = G * _log_int(rng, 1, 16 // G)
    P = rng.choice((16, 32, 48, 64, 64, 64, 128))
    N = rng.choice((16, 24, 32, 64, 64, 64, 128))
    if op == "step":
        B = _log_int(rng, 1, min(256, STEP_WORK // (H * P * N)))
        return _case(None, op, B, 1, "score", kind, B > 1 and rng.random() < 0.5, H=H, P=P, G=G, N=N,
                     W=rng.choice((2, 3, 4, 4)))
    # float32 products and small heads cost more for each element than the listed cases' do
    share = {"float32": 8, "float16": 3, "bfloat16": 1}[kind]
    most = min(SCAN_WORK // (share * H * max(P, 64) * max(N, 64)), TRAIN_TOKENS // (H * P + 2 * G * N))
    B = _log_int(rng, 1, min(64, most))
    T = _log_int(rng, 1, min(100_000, most // B))
    return _case(None, op, B, T, mode, kind, B > 1 and rng.random() < 0.6, H=H, P=P, G=G, N=N)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    dev = "cuda"
    op, B, T, train = case["op"], case["B"], case["T"], case["mode"] == "train"
    dtype = DTYPES[case["type"]]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=dev)  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, generator=g, device=dev)  # noqa: E731
    s = {"op": op, "train": train, "dtype": dtype, "lengths": None}
    if op == "step":
        # tokens each stream has seen; idle slots hold -1
        seen = torch.randint(0, 5000, (B,), generator=g, device=dev, dtype=torch.int32)
        if case["ragged"]:
            seen = torch.where(uniform(B) < 0.1, torch.full_like(seen, -1), seen)
        s["seen"] = seen
    elif case["ragged"]:
        lengths = torch.randint((T + 1) // 2, T + 1, (B,), generator=g, device=dev, dtype=torch.int32)
        lengths[B // 2] = 0
        s["lengths"] = lengths
    if op == "embed":
        V, D = case["V"], case["D"]
        r = uniform(B, T)
        tokens = (r ** 4 * V if case["skew"] else r * V).to(torch.int32).clamp_(max=V - 1)
        s.update(tokens=tokens, table=normal(V, D), scale=math.sqrt(D))
        s["table"] = s["table"].to(dtype)
        if train:
            s["grad"] = (normal(B, T, D) * 0.1).to(dtype)
        return s
    W = case.get("W")
    if op == "conv":
        C = case["C"]
        s.update(u=normal(B, T, C).to(dtype), weight=normal(C, W) / math.sqrt(W), bias=0.1 * normal(C))
        if train:
            s["grad"] = (normal(B, T, C) * 0.1).to(dtype)
        return s
    H, P, G, N = (case[k] for k in "HPGN")
    width = H * P + 2 * G * N
    s["sizes"] = (H, P, G, N)
    # step sizes between 1e-3 and 1e-1 where dt is 0, rates between 1 and 16: memories of one to a thousand tokens
    start = torch.exp(uniform(H) * math.log(100.0) + math.log(1e-3))
    s.update(dt_bias=start + torch.log(-torch.expm1(-start)), rate=-(1.0 + 15.0 * uniform(H)), skip=normal(H))
    state = 0.5 * normal(B, H, P, N)
    if op == "step":
        # the input projection's output: a gate in front, x, B and C, then dt
        row = torch.cat([normal(B, H * P + width), 0.5 * normal(B, H)], 1).to(dtype)
        s.update(u=row[:, H * P:H * P + width], dt=row[:, H * P + width:], state=state,
                 weight=normal(width, W) / math.sqrt(W), bias=0.1 * normal(width),
                 ring=normal(B, width, W).to(dtype))
        s["state_out"] = torch.empty_like(s["state"])
        s["ring_out"] = torch.empty_like(s["ring"])
        s["y"] = torch.empty(B, H * P, device=dev, dtype=dtype)
        return s
    # what the convolution leaves: x, B and C side by side
    v = normal(B, T, width)
    xbc = (v * torch.sigmoid(v)).to(dtype)
    del v
    dt = (0.5 * normal(B, T, H)).to(dtype)
    if s["lengths"] is not None:
        # what lies behind a sequence's end is not a number
        past = torch.arange(T, device=dev)[None, :] >= s["lengths"][:, None]
        xbc.masked_fill_(past[:, :, None], float("nan"))
        dt.masked_fill_(past[:, :, None], float("nan"))
    s.update(xbc=xbc, dt=dt, state=None if train else state)
    if train:
        s["grad"] = (0.1 * normal(B, T, H * P)).to(dtype)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _silu(a):
    return a * torch.sigmoid(a)


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))


def _valid(s, B, T):
    t = torch.arange(T, device="cuda")
    if s["lengths"] is None:
        return torch.ones(B, T, dtype=torch.bool, device="cuda")
    return t[None, :] < s["lengths"][:, None]


def _plain_embed(s):
    tokens, table = s["tokens"], s["table"]
    B, T = tokens.shape
    valid = _valid(s, B, T)
    out = (table[tokens.long()].float() * s["scale"]).masked_fill(~valid[:, :, None], 0.0).to(s["dtype"])
    if not s["train"]:
        return (out,)
    g = s["grad"].float().masked_fill(~valid[:, :, None], 0.0) * s["scale"]
    grad_table = torch.zeros(table.shape, device="cuda")
    grad_table.index_add_(0, tokens.reshape(-1).long(), g.reshape(B * T, -1))
    return out, grad_table


def _plain_conv_rows(u, weight, bias):
    W, T = weight.shape[1], u.shape[1]
    padded = torch.nn.functional.pad(u, (0, 0, W - 1, 0))
    a = bias.expand_as(u)
    for j in range(W):
        a = a + weight[:, j] * padded[:, j:j + T]
    return _silu(a)


def _plain_conv(s):
    B, T, C = s["u"].shape
    past = ~_valid(s, B, T)[:, :, None]
    with torch.set_grad_enabled(s["train"]):
        u, weight, bias = s["u"].float().masked_fill(past, 0.0), s["weight"], s["bias"]
        if s["train"]:
            u, weight, bias = (v.detach().requires_grad_() for v in (u, weight, bias))
        out = _plain_conv_rows(u, weight, bias).masked_fill(past, 0.0)
        y = out.detach().to(s["dtype"])
        if not s["train"]:
            return (y,)
        gu, gw, gb = torch.autograd.grad(out, (u, weight, bias), s["grad"].float().masked_fill(past, 0.0))
    return y, gu.to(s["dtype"]), gw, gb


def _plain_scan_rows(xbc, dt, rate, skip, dt_bias, state, valid, sizes):
    """Chunks of CHUNK positions: products within a chunk, the state from chunk to chunk."""
    H, P, G, N = sizes
    B, T, _ = xbc.shape
    pad = -T % CHUNK
    n = (T + pad) // CHUNK
    delta = _softplus(dt + dt_bias).masked_fill(~valid[:, :, None], 0.0)
    if pad:
        xbc = torch.nn.functional.pad(xbc, (0, 0, 0, pad))
        delta = torch.nn.functional.pad(delta, (0, 0, 0, pad))
    x = xbc[..., :H * P].reshape(B, n, CHUNK, H, P).transpose(2, 3)
    b = xbc[..., H * P:H * P + G * N].reshape(B, n, CHUNK, G, N).transpose(2, 3)
    c = xbc[..., H * P + G * N:].reshape(B, n, CHUNK, G, N).transpose(2, 3)
    delta = delta.reshape(B, n, CHUNK, H).transpose(2, 3)                       # [B, n, H, CHUNK]
    gone = (delta * rate[:, None]).cumsum(3)
    later = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").triu(1)
    decay = torch.exp((gone[..., :, None] - gone[..., None, :]).masked_fill(later, -math.inf))
    heads = lambda v: v[:, :, :, None].expand(B, n, G, H // G, *v.shape[3:]).reshape(B, n, H, *v.shape[3:])  # noqa: E731
    u = x * delta[..., None]
    y = torch.matmul(heads(torch.matmul(c, b.transpose(3, 4))) * decay, u)
    carried = torch.exp(gone[..., -1:] - gone)
    added = torch.matmul((u * carried[..., None]).transpose(3, 4), heads(b))    # [B, n, H, P, N]
    kept = torch.exp(gone[..., -1])[..., None, None]
    # states before each chunk and after the last: a scan by doubling over the chunks
    first = torch.zeros(B, 1, H, P, N, device="cuda") if state is None else state[:, None]
    h, kept = torch.cat([first, added], 1), torch.nn.functional.pad(kept, (0, 0, 0, 0, 0, 0, 1, 0))
    reach = 1
    while reach <= n:
        h = torch.cat([h[:, :reach], h[:, reach:] + kept[:, reach:] * h[:, :-reach]], 1)
        kept = torch.cat([kept[:, :reach], kept[:, reach:] * kept[:, :-reach]], 1)
        reach *= 2
    y = y + torch.exp(gone)[..., None] * torch.matmul(heads(c), h[:, :-1].transpose(3, 4))
    y = y + skip[:, None, None] * x
    y = y.transpose(2, 3).reshape(B, n * CHUNK, H * P)[:, :T]
    return y.masked_fill(~valid[:, :, None], 0.0), h[:, -1]


def _plain_scan(s):
    B, T, _ = s["xbc"].shape
    valid = _valid(s, B, T)
    past = ~valid[:, :, None]
    with torch.set_grad_enabled(s["train"]):
        xbc, dt = s["xbc"].float().masked_fill(past, 0.0), s["dt"].float().masked_fill(past, 0.0)
        leaves = [xbc, dt, s["rate"], s["skip"], s["dt_bias"]]
        if s["train"]:
            leaves = [v.detach().requires_grad_() for v in leaves]
        y, h = _plain_scan_rows(*leaves, s["state"], valid, s["sizes"])
        out = y.detach().to(s["dtype"])
        if not s["train"]:
            return out, h
        grads = torch.autograd.grad(y, leaves, s["grad"].float().masked_fill(past, 0.0))
    return (out, grads[0].to(s["dtype"]), grads[1].to(s["dtype"])) + grads[2:]


def _plain_step(s):
    H, P, G, N = s["sizes"]
    u, seen, W = s["u"].float(), s["seen"].long(), s["weight"].shape[1]
    B = u.shape[0]
    live = seen >= 0
    ring = s["ring"].clone()
    rows = torch.arange(B, device="cuda")
    slot = seen.clamp(min=0) % W
    ring[rows, :, slot] = torch.where(live[:, None], s["u"], ring[rows, :, slot])
    a = s["bias"] + s["weight"][:, W - 1] * u
    for j in range(1, W):
        before = seen - j
        past = ring[rows, :, before.clamp(min=0) % W].float()
        a = a + s["weight"][:, W - 1 - j] * torch.where((before >= 0)[:, None], past, torch.zeros_like(past))
    a = _silu(a)
    x = a[:, :H * P].reshape(B, H, P)
    b = a[:, H * P:H * P + G * N].reshape(B, G, 1, N).expand(B, G, H // G, N).reshape(B, H, N)
    c = a[:, H * P + G * N:].reshape(B, G, 1, N).expand(B, G, H // G, N).reshape(B, H, N)
    delta = _softplus(s["dt"].float() + s["dt_bias"])
    h = s["state"] * torch.exp(delta * s["rate"])[:, :, None, None] + (delta[:, :, None] * x)[..., None] * b[:, :, None]
    y = torch.matmul(h, c[..., None])[..., 0] + s["skip"][:, None] * x
    h = torch.where(live[:, None, None, None], h, s["state"])
    y = torch.where(live[:, None, None], y, torch.zeros_like(y)).reshape(B, H * P).to(s["dtype"])
    return y, h, ring


# ---- the library's operators ----------------------------------------------------------------------------------------

def _own(s):
    from paper_2604_18780_amd import binding as sb
    op, lengths = s["op"], s["lengths"]
    if op == "embed":
        out = sb.semicrf_embed_fwd(s["tokens"], s["table"], s["scale"], lengths)
        if not s["train"]:
            return (out,)
        return out, sb.semicrf_embed_bwd(s["tokens"], s["grad"], s["table"].shape[0], s["scale"], lengths)
    if op == "conv":
        out = sb.semicrf_conv_fwd(s["u"], s["weight"], s["bias"], lengths)
        if not s["train"]:
            return (out,)
        return (out,) + sb.semicrf_conv_bwd(s["u"], s["weight"], s["bias"], s["grad"], lengths)
    if op == "step":
        sb.semicrf_ssm_step(s["u"], s["weight"], s["bias"], s["dt"], s["rate"], s["skip"], s["dt_bias"], s["seen"],
                            s["ring"], s["state"], groups=s["sizes"][2], out=(s["y"], s["ring_out"], s["state_out"]))
        return s["y"], s["state_out"], s["ring_out"]
    H, P, G, N = s["sizes"]
    B, T, _ = s["xbc"].shape
    x = s["xbc"][..., :H * P].unflatten(2, (H, P))
    b = s["xbc"][..., H * P:H * P + G * N].unflatten(2, (G, N))
    c = s["xbc"][..., H * P + G * N:].unflatten(2, (G, N))
    y, h = sb.semicrf_ssm_fwd(x, b, c, s["dt"], s["rate"], s["skip"], s["dt_bias"], lengths, s["state"],
                              want_state=not s["train"])
    y = y.view(B, T, H * P)
    if not s["train"]:
        return y, h
    g = sb.semicrf_ssm_bwd(x, b, c, s["dt"], s["rate"], s["skip"], s["dt_bias"], s["grad"].view(B, T, H, P), lengths)
    return y, g["grad_xbc"], g["grad_dt"], g["grad_rate"], g["grad_skip"], g["grad_dt_bias"]


def run(s):
    if own:
        return _own(s)
    return {"embed": _plain_embed, "conv": _plain_conv, "scan": _plain_scan, "step": _plain_step}[s["op"]](s)


# ---- 64 bits, from the definitions ----------------------------------------------------------------------------------

def _exact_embed(s):
    B, T = s["tokens"].shape
    V, D = s["table"].shape
    out = torch.zeros(B, T, D, dtype=torch.float64, device="cuda")
    grad_table = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for i in range(B):
        L = T if s["lengths"] is None else int(s["lengths"][i])
        ids = s["tokens"][i, :L].long()
        out[i, :L] = s["table"].double()[ids] * s["scale"]
        if s["train"]:
            grad_table.index_add_(0, ids, s["grad"][i, :L].double() * s["scale"])
    return (out, grad_table) if s["train"] else (out,)


def _exact_conv(s):
    u, w, bias = s["u"].double(), s["weight"].double(), s["bias"].double()
    B, T, C = u.shape
    W = w.shape[1]
    out, gu = torch.zeros_like(u), torch.zeros_like(u)
    gw, gb = torch.zeros_like(w), torch.zeros_like(bias)
    for i in range(B):
        L = T if s["lengths"] is None else int(s["lengths"][i])
        if L == 0:
            continue
        a = bias.repeat(L, 1)
        for back in range(min(W, L)):
            a[back:] += w[:, W - 1 - back] * u[i, :L - back]
        sg = 1.0 / (1.0 + torch.exp(-a))
        out[i, :L] = a * sg
        if not s["train"]:
            continue
        da = s["grad"][i, :L].double() * sg * (1.0 + a * (1.0 - sg))
        gb += da.sum(0)
        for back in range(min(W, L)):
            gu[i, :L - back] += w[:, W - 1 - back] * da[back:]
            gw[:, W - 1 - back] += (da[back:] * u[i, :L - back]).sum(0)
    return (out, gu, gw, gb) if s["train"] else (out,)


def _exact_scan(s):
    """Every pair of positions at once: y = (decay * C B^T) u, and the gradients of that product."""
    H, P, G, N = s["sizes"]
    B, T, width = s["xbc"].shape
    f64 = dict(dtype=torch.float64, device="cuda")
    y, gxbc, gdt = torch.zeros(B, T, H * P, **f64), torch.zeros(B, T, width, **f64), torch.zeros(B, T, H, **f64)
    last = torch.zeros(B, H, P, N, **f64) if s["state"] is None else s["state"].double()
    grate, gskip, gbias = (torch.zeros(H, **f64) for _ in range(3))
    rate, skip = s["rate"].double(), s["skip"].double()
    for i in range(B):
        L = T if s["lengths"] is None else int(s["lengths"][i])
        if L == 0:
            continue
        raw = s["dt"][i, :L].double() + s["dt_bias"].double()
        delta = torch.where(raw > 30, raw, torch.log1p(torch.exp(torch.clamp(raw, max=30))))
        later = torch.ones(L, L, dtype=torch.bool, device="cuda").triu(1)
        for h in range(H):
            grp = h // (H // G)
            x = s["xbc"][i, :L, h * P:(h + 1) * P].double()
            at_b, at_c = H * P + grp * N, H * P + (G + grp) * N
            b, c = s["xbc"][i, :L, at_b:at_b + N].double(), s["xbc"][i, :L, at_c:at_c + N].double()
            d = delta[:, h]
            gone = torch.cumsum(d * rate[h], 0)
            decay = torch.exp((gone[:, None] - gone[None, :]).masked_fill(later, -math.inf))
            u = d[:, None] * x
            pairs = decay * (c @ b.T)
            y[i, :L, h * P:(h + 1) * P] = pairs @ u + skip[h] * x
            if not s["train"]:
                y[i, :L, h * P:(h + 1) * P] += torch.exp(gone)[:, None] * (c @ last[i, h].T)
                last[i, h] = last[i, h] * torch.exp(gone[-1]) + (u * torch.exp(gone[-1] - gone)[:, None]).T @ b
                continue
            dy = s["grad"][i, :L, h * P:(h + 1) * P].double()
            dpairs = dy @ u.T
            du = pairs.T @ dy
            gxbc[i, :L, h * P:(h + 1) * P] = d[:, None] * du + skip[h] * dy
            gxbc[i, :L, at_c:at_c + N] += (dpairs * decay) @ b
            gxbc[i, :L, at_b:at_b + N] += (dpairs * decay).T @ c
            # decay[i,j] holds the steps j+1..i: step t lies in every pair with j < t <= i
            weighed = dpairs * pairs
            dgone = weighed.sum(1) - weighed.sum(0)
            dstep = torch.flip(torch.cumsum(torch.flip(dgone, (0,)), 0), (0,))
            grate[h] += (dstep * d).sum()
            gskip[h] += (dy * x).sum()
            ddelta = dstep * rate[h] + (du * x).sum(1)
            gdt[i, :L, h] = ddelta / (1.0 + torch.exp(-raw[:, h]))
            gbias[h] += gdt[i, :L, h].sum()
    return (y, gxbc, gdt, grate, gskip, gbias) if s["train"] else (y, last)


def _exact_step(s):
    H, P, G, N = s["sizes"]
    B, width, W = s["ring"].shape
    y = torch.zeros(B, H * P, dtype=torch.float64)
    state, ring = s["state"].double().cpu(), s["ring"].double().cpu()
    u, w, bias, dt = (s[k].double().cpu() for k in ("u", "weight", "bias", "dt"))
    rate, skip, dt_bias, seen = (s[k].double().cpu() for k in ("rate", "skip", "dt_bias", "seen"))
    for i in range(B):
        n = int(seen[i])
        if n < 0:
            continue
        ring[i, :, n % W] = u[i]
        a = bias.clone()
        for back in range(min(W, n + 1)):
            a += w[:, W - 1 - back] * ring[i, :, (n - back) % W]
        a = a / (1.0 + torch.exp(-a))
        for h in range(H):
            grp = h // (H // G)
            x = a[h * P:(h + 1) * P]
            b = a[H * P + grp * N:H * P + (grp + 1) * N]
            c = a[H * P + (G + grp) * N:H * P + (G + grp + 1) * N]
            d = torch.log1p(torch.exp(dt[i, h] + dt_bias[h]))
            state[i, h] = state[i, h] * torch.exp(d * rate[h]) + d * torch.outer(x, b)
            y[i, h * P:(h + 1) * P] = state[i, h] @ c + skip[h] * x
    return y, state, ring


def exact(case, seed):
    tokens = case["B"] * case["T"]
    if case["op"] == "scan" and tokens * case["T"] * case["H"] > 2e9:
        return None
    if tokens * case.get("C", case.get("D", 0)) > 3e8:
        return None
    s = prepare(case, seed)
    return {"embed": _exact_embed, "conv": _exact_conv, "scan": _exact_scan, "step": _exact_step}[s["op"]](s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    """Bytes: every input and output once.  Flops: the recurrence itself for the scans (a state entry is scaled, added to
    and read once for each token; the gradients need that again and as much backwards), one multiply-add for each tap."""
    op, B, T, train, e = case["op"], case["B"], case["T"], case["mode"] == "train", BYTES[case["type"]]
    share = 0.75 * (B - 1) / B if case["ragged"] and op != "step" else 1.0
    rows, valid = B * T, share * B * T
    if op == "embed":
        V, D = case["V"], case["D"]
        read = 4 * valid + min(V, valid) * D * e
        if not train:
            return {"bytes": float(read + rows * D * e), "flops": float(valid * D)}
        return {"bytes": float(read + rows * D * e + valid * D * e + V * D * 4), "flops": float(3 * valid * D)}
    if op == "conv":
        C, W = case["C"], case["W"]
        if not train:
            return {"bytes": float((valid + rows) * C * e), "flops": float(valid * C * 2 * W)}
        return {"bytes": float((2 * valid + 2 * rows) * C * e), "flops": float(valid * C * 6 * W)}
    H, P, G, N = (case[k] for k in "HPGN")
    width, state = H * P + 2 * G * N, B * H * P * N
    if op == "step":
        live = 0.9 if case["ragged"] else 1.0
        row = B * (width + H + H * P) * e + 2 * B * width * case["W"] * e + width * case["W"] * 4
        return {"bytes": float(8 * state + row), "flops": float(5 * live * state)}
    cells = valid * H * P * N
    if not train:
        return {"bytes": float((valid * (width + H) + rows * H * P) * e + 8 * state), "flops": float(5 * cells)}
    moved = valid * (width + H + H * P) + rows * (H * P + width + H)
    return {"bytes": float(moved * e), "flops": float(14 * cells)}
