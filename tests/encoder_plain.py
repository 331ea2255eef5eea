"""Plain 64-bit forms of the encoder operators, one token at a time, for the tests: embedding, short causal convolution,
selective state space scan, and the gradients of the three by the recurrences' own derivatives."""
import numpy as np


def sigmoid(v):
    return np.where(v >= 0, 1.0 / (1.0 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1.0 + np.exp(-np.abs(v))))


def softplus(v):
    return np.maximum(v, 0.0) + np.log1p(np.exp(-np.abs(v)))


def embed(tokens, table, scale, lengths):
    B, T = tokens.shape
    out = np.zeros((B, T, table.shape[1]))
    for b in range(B):
        for t in range(lengths[b]):
            if 0 <= tokens[b, t] < len(table):
                out[b, t] = scale * table[tokens[b, t]]
    return out


def embed_grad(tokens, grad, V, scale, lengths):
    g = np.zeros((V, grad.shape[2]))
    for b in range(tokens.shape[0]):
        for t in range(lengths[b]):
            if 0 <= tokens[b, t] < V:
                g[tokens[b, t]] += scale * grad[b, t]
    return g


def conv(u, weight, bias, lengths, linear=False, ring=None, seen=None):
    """Returns (out, ring after the call)."""
    B, T, C = u.shape
    W = weight.shape[1]
    out = np.zeros((B, T, C))
    ring = np.zeros((B, C, W)) if ring is None else ring.copy()
    for b in range(B):
        n = 0 if seen is None else seen[b]
        if n < 0:
            continue
        for t in range(lengths[b]):
            p = n + t
            ring[b, :, p % W] = u[b, t]
            a = bias.copy()
            for back in range(W):
                if p - back >= 0:
                    a += weight[:, W - 1 - back] * ring[b, :, (p - back) % W]
            out[b, t] = a if linear else a * sigmoid(a)
    return out, ring


def conv_grad(u, weight, bias, grad, lengths, linear=False):
    B, T, C = u.shape
    W = weight.shape[1]
    gu, gw, gb = np.zeros_like(u), np.zeros_like(weight), np.zeros_like(bias)
    for b in range(B):
        for t in range(lengths[b]):
            a = bias.copy()
            for back in range(min(W, t + 1)):
                a += weight[:, W - 1 - back] * u[b, t - back]
            s = sigmoid(a)
            da = grad[b, t] * (1.0 if linear else s * (1.0 + a * (1.0 - s)))
            gb += da
            for back in range(min(W, t + 1)):
                gw[:, W - 1 - back] += da * u[b, t - back]
                gu[b, t - back] += da * weight[:, W - 1 - back]
    return gu, gw, gb


def scan(x, b, c, dt, rate, skip, dt_bias, lengths, state):
    """x [B,T,H,P], b, c [B,T,G,N], dt [B,T,H], state [B,H,P,N].  Returns (y, last state, states before each token)."""
    B, T, H, P = x.shape
    G = b.shape[2]
    y, last = np.zeros_like(x), state.copy()
    before = np.zeros((B, T) + state.shape[1:])
    grp = np.arange(H) // (H // G)
    for i in range(B):
        h = state[i].copy()
        for t in range(lengths[i]):
            before[i, t] = h
            d = softplus(dt[i, t] + dt_bias)
            h = np.exp(d * rate)[:, None, None] * h + (d[:, None] * x[i, t])[:, :, None] * b[i, t][grp][:, None, :]
            y[i, t] = np.einsum("hpn,hn->hp", h, c[i, t][grp]) + skip[:, None] * x[i, t]
        last[i] = h
    return y, last, before


def scan_grad(x, b, c, dt, rate, skip, dt_bias, lengths, state, gy, glast):
    B, T, H, P = x.shape
    G = b.shape[2]
    _, _, before = scan(x, b, c, dt, rate, skip, dt_bias, lengths, state)
    grp = np.arange(H) // (H // G)
    out = dict(grad_x=np.zeros_like(x), grad_b=np.zeros_like(b), grad_c=np.zeros_like(c), grad_dt=np.zeros_like(dt),
               grad_rate=np.zeros(H), grad_skip=np.zeros(H), grad_dt_bias=np.zeros(H), grad_state=np.zeros_like(state))
    for i in range(B):
        g = glast[i].copy()
        for t in range(lengths[i] - 1, -1, -1):
            raw = dt[i, t] + dt_bias
            d = softplus(raw)
            keep = np.exp(d * rate)
            bt, ct = b[i, t][grp], c[i, t][grp]
            h = keep[:, None, None] * before[i, t] + (d[:, None] * x[i, t])[:, :, None] * bt[:, None, :]
            np.add.at(out["grad_c"][i, t], grp, np.einsum("hpn,hp->hn", h, gy[i, t]))
            g = g + gy[i, t][:, :, None] * ct[:, None, :]
            du = np.einsum("hpn,hn->hp", g, bt)
            np.add.at(out["grad_b"][i, t], grp, np.einsum("hpn,hp->hn", g, d[:, None] * x[i, t]))
            out["grad_x"][i, t] = d[:, None] * du + skip[:, None] * gy[i, t]
            out["grad_skip"] += (x[i, t] * gy[i, t]).sum(1)
            dl = (g * keep[:, None, None] * before[i, t]).sum((1, 2))
            gdt = ((x[i, t] * du).sum(1) + rate * dl) * sigmoid(raw)
            out["grad_rate"] += d * dl
            out["grad_dt"][i, t] = gdt
            out["grad_dt_bias"] += gdt
            g = keep[:, None, None] * g
        out["grad_state"][i] = g
    return out
