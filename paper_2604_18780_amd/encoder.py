"""A segment model from tokens to log-partition: embedding, selective state space encoder, semi-CRF.

    tokens -> embedding -> projection -> short convolution -> selective scan -> projection -> emissions -> semi-CRF

Everything that is not a plain matrix product runs in the library: ``Encoder.emissions`` and ``Encoder.backward`` are the two
directions over whole sequences, ``Stream`` is the same encoder one token at a time.  ``python -m
paper_2604_18780_amd.encoder`` trains one on a synthetic text whose segments differ in what they draw their tokens from, then
annotates a stream token by token.
"""
from __future__ import annotations

import torch

from . import binding as sb


class Encoder:
    """Parameters are float32; products and activations are in `dtype`."""

    def __init__(self, vocabulary, labels, width=64, heads=4, channels=32, groups=1, states=32, taps=4,
                 dtype=torch.bfloat16, device="cuda:0", seed=0):
        H, P, G, N = heads, channels, groups, states
        self.sizes, self.dtype, self.scale = (H, P, G, N), dtype, width ** 0.5
        # x, B and C side by side, as the convolution and the scan take them, then dt; rows end on 16 bytes
        self.columns, self.row = H * P + 2 * G * N, H * P + 2 * G * N + (H + 7) // 8 * 8
        g = torch.Generator().manual_seed(seed)
        normal = lambda *s, sd: sd * torch.randn(*s, generator=g)  # noqa: E731
        delta = torch.exp(torch.rand(H, generator=g) * 4.6 - 6.9)  # steps between 1e-3 and 1e-1
        self.params = {k: v.to(device) for k, v in dict(
            table=normal(vocabulary, width, sd=width ** -0.5), w_in=normal(width, self.row, sd=width ** -0.5),
            taps=normal(self.columns, taps, sd=taps ** -0.5), taps_bias=torch.zeros(self.columns),
            log_rate=torch.log(1.0 + 15.0 * torch.rand(H, generator=g)), skip=torch.ones(H),
            dt_bias=delta + torch.log(-torch.expm1(-delta)), w_out=normal(H * P, labels, sd=(H * P) ** -0.5)).items()}

    def split(self, v):
        """Views of x, B and C in rows of the convolution's channels."""
        H, P, G, N = self.sizes
        x, b, c = v.split((H * P, G * N, G * N), dim=-1)
        return x.unflatten(-1, (H, P)), b.unflatten(-1, (G, N)), c.unflatten(-1, (G, N))

    def emissions(self, tokens, lengths=None):
        """tokens [B,T] int32 -> emission scores [B,T,labels] in float32, and what `backward` needs."""
        p, dt = self.params, self.dtype
        H, P, _, _ = self.sizes
        e = sb.semicrf_embed_fwd(tokens, p["table"].to(dt), self.scale, lengths)
        z = e @ p["w_in"].to(dt)
        u, steps = z[..., :self.columns], z[..., self.columns:self.columns + H]
        v = sb.semicrf_conv_fwd(u, p["taps"], p["taps_bias"], lengths)
        y, _ = sb.semicrf_ssm_fwd(*self.split(v), steps, -torch.exp(p["log_rate"]), p["skip"], p["dt_bias"], lengths,
                                  want_state=False)
        y = y.flatten(2)
        return (y @ p["w_out"].to(dt)).float(), (tokens, lengths, e, z, v, y)

    def backward(self, saved, grad_emis):
        """Gradients of all parameters from that of the emission scores."""
        tokens, lengths, e, z, v, y = saved
        p, dt = self.params, self.dtype
        H, P, G, N = self.sizes
        rows = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
        ge = grad_emis.to(dt)
        gy = ge @ p["w_out"].to(dt).t()
        rate = -torch.exp(p["log_rate"])
        s = sb.semicrf_ssm_bwd(*self.split(v), z[..., self.columns:self.columns + H], rate, p["skip"], p["dt_bias"],
                               gy.unflatten(2, (H, P)), lengths)
        gz = torch.zeros_like(z)
        gz[..., self.columns:self.columns + H] = s["grad_dt"]
        _, taps, taps_bias = sb.semicrf_conv_bwd(z[..., :self.columns], p["taps"], p["taps_bias"], s["grad_xbc"], lengths,
                                                 grad_u=gz[..., :self.columns])
        table = sb.semicrf_embed_bwd(tokens, gz @ p["w_in"].to(dt).t(), p["table"].shape[0], self.scale, lengths)
        return dict(table=table, w_in=(rows(e).t() @ rows(gz)).float(), taps=taps, taps_bias=taps_bias,
                    log_rate=s["grad_rate"] * rate, skip=s["grad_skip"], dt_bias=s["grad_dt_bias"],
                    w_out=(rows(y).t() @ rows(ge)).float())


class Stream:
    """The encoder one token at a time, for `streams` texts side by side; `seen` < 0 marks one that is idle.  Its parameters are the
    encoder's of when it was made, or of the last `refresh`: laid out once, not for every token."""

    def __init__(self, encoder, streams):
        self.enc = encoder
        p = encoder.params
        H, P, _, N = encoder.sizes
        device = p["table"].device
        self.seen = torch.zeros(streams, dtype=torch.int32, device=device)
        self.ring = torch.zeros(streams, *p["taps"].shape, dtype=encoder.dtype, device=device)
        self.state = torch.zeros(streams, H, P, N, device=device)
        self.refresh()

    def refresh(self):
        """Takes the encoder's parameters as they are now; texts go on."""
        p = self.enc.params
        self.params = {k: p[k].to(self.enc.dtype, copy=True) for k in ("table", "w_in", "w_out")}
        self.params.update({k: p[k].clone() for k in ("taps", "taps_bias", "skip", "dt_bias")}, rate=-torch.exp(p["log_rate"]))

    def step(self, tokens):
        """tokens [streams] int32 -> emission scores [streams,labels] of these positions."""
        enc, p = self.enc, self.params
        H, _, G, _ = enc.sizes
        z = sb.semicrf_embed_fwd(tokens[:, None], p["table"], enc.scale)[:, 0] @ p["w_in"]
        y = sb.semicrf_ssm_step(z[:, :enc.columns], p["taps"], p["taps_bias"], z[:, enc.columns:enc.columns + H], p["rate"],
                                p["skip"], p["dt_bias"], self.seen, self.ring, self.state, groups=G)
        self.seen += (self.seen >= 0).int()
        return (y @ p["w_out"]).float()


def gold(labels, lengths, emis, crf):
    """Score of the segmentations that labels [B,T] stand for (a segment ends where the label changes, or after K positions), summed
    over sequences, and its gradients by emissions, transitions and durations.  A first segment is entered from any label."""
    B, T = labels.shape
    K, C = crf["dur"].shape
    t = torch.arange(T, device=labels.device).expand(B, T)
    last = lengths[:, None] - 1
    change = torch.ones_like(labels, dtype=torch.bool)
    change[:, 1:] = labels[:, 1:] != labels[:, :-1]
    since = (t - torch.where(change, t, 0).cummax(1).values) % K  # positions of the segment before this one
    begins, valid = since == 0, t <= last
    ends = valid & (torch.cat([begins[:, 1:], begins[:, :1]], 1) | (t == last))
    emission = torch.zeros_like(emis).scatter_(2, labels[..., None], valid[..., None].float())
    duration = torch.zeros_like(crf["dur"]).index_put_((since[ends], labels[ends]), emis.new_ones(()), accumulate=True)
    move = torch.zeros_like(crf["trans"])
    inner = (begins & valid)[:, 1:]
    move.index_put_((labels[:, :-1][inner], labels[:, 1:][inner]), emis.new_ones(()), accumulate=True)
    entered = labels[:, 0][lengths > 0]
    score = (emission * emis).sum() + (duration * crf["dur"]).sum() + (move * crf["trans"]).sum() \
        + torch.logsumexp(crf["trans"], 0)[entered].sum()
    move.index_add_(1, entered, torch.softmax(crf["trans"], 0)[:, entered])
    return score, dict(emis=emission, trans=move, dur=duration)


def loss_and_gradients(encoder, crf, tokens, lengths, labels):
    """Mean negative log-likelihood of the labels' segmentations, and its gradients by the parameters of the encoder and of the
    semi-CRF (crf: trans [C,C] and dur [K,C])."""
    B = tokens.shape[0]
    emis, saved = encoder.emissions(tokens, lengths)
    logz, g_emis, g_trans, g_dur, _ = sb.semicrf_fwd_bwd(emis, lengths, crf["trans"], crf["dur"], flags=0, want_pos_marg=False)
    score, counts = gold(labels, lengths, emis, crf)
    grads = encoder.backward(saved, (g_emis - counts["emis"]) / B)
    grads.update(trans=(g_trans - counts["trans"]) / B, dur=(g_dur - counts["dur"]) / B)
    return (logz.sum() - score) / B, grads


def synthetic(B, T, vocabulary, labels, mean, device, seed):
    """Texts whose segments (geometric lengths) draw their tokens from overlapping ranges of the vocabulary, one for each label."""
    g = torch.Generator().manual_seed(seed)
    change = torch.rand(B, T, generator=g) < 1.0 / mean
    hop = torch.where(change, torch.randint(1, labels, (B, T), generator=g), torch.zeros(B, T, dtype=torch.long))
    label = hop.cumsum(1) % labels
    span = 2 * vocabulary // (labels + 1)
    token = label * (vocabulary // (labels + 1)) + torch.randint(0, span, (B, T), generator=g)
    lengths = torch.randint(T // 2, T + 1, (B,), generator=g, dtype=torch.int32)
    return token.int().to(device), lengths.to(device), label.to(device)


def main(B=64, T=256, K=16, C=24, vocabulary=256, steps=60, device="cuda:0"):
    enc = Encoder(vocabulary, C, width=64, heads=4, channels=32, states=32, device=device)
    crf = dict(trans=torch.zeros(C, C, device=device), dur=torch.zeros(K, C, device=device))
    everything = {**enc.params, **crf}
    optimizer = torch.optim.Adam(everything.values(), lr=1e-2)
    for step in range(steps):
        tokens, lengths, labels = synthetic(B, T, vocabulary, C, 6.0, device, seed=step)
        loss, grads = loss_and_gradients(enc, crf, tokens, lengths, labels)
        for k, v in grads.items():
            everything[k].grad = v
        optimizer.step()
        if step % 10 == 0 or step == steps - 1:
            print("step %3d  loss per position %.4f" % (step, loss.item() * B / lengths.sum().item()), flush=True)

    tokens, lengths, labels = synthetic(4, 64, vocabulary, C, 6.0, device, seed=steps)
    whole, _ = enc.emissions(tokens)
    stream = Stream(enc, 4)
    worst = 0.0
    for t in range(tokens.shape[1]):
        worst = max(worst, (stream.step(tokens[:, t].contiguous()) - whole[:, t]).abs().max().item())
    print("64 tokens of 4 streams one at a time: emissions within %.3f of the whole texts' (largest %.1f)"
          % (worst, whole.abs().max().item()))
    full = torch.full((4,), 64, dtype=torch.int32, device=device)
    decoded = sb.semicrf_viterbi(whole, full, crf["trans"], crf["dur"], flags=0)
    print("best segmentations' scores:", [round(v, 1) for v in decoded[0].tolist()])
    return loss


if __name__ == "__main__":
    main()
