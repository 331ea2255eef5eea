"""GPU tests of the model that runs embedding, convolution, scan and semi-CRF together.

The loss's gradients against central differences of the whole model in 64 bits (plain recurrences, and the CPU oracle for the
log-partition).  The semi-CRF's gradients are float32 of values up to 1, right to 1e-5 of their norm, and so is what the
encoder makes of them in float32: 5e-5 of the two norms bounds their product with a direction.  A stream and a whole text in
float32 differ by the order of sums: 1e-4 of the largest emission."""
import numpy as np
import pytest
import torch

import encoder_plain as plain
import oracle
from paper_2604_18780_amd import encoder

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def model(dtype=torch.float32, labels=3, K=5):
    enc = encoder.Encoder(11, labels, width=16, heads=4, channels=8, groups=2, states=8, dtype=dtype, device=DEV, seed=1)
    g = torch.Generator().manual_seed(2)
    crf = dict(trans=(0.3 * torch.randn(labels, labels, generator=g)).to(DEV),
               dur=(0.3 * torch.randn(K, labels, generator=g)).to(DEV))
    return enc, crf


def loss64(enc, p, tokens, lengths, labels):
    """The mean negative log-likelihood in 64 bits, segment by segment."""
    H, P, G, N = enc.sizes
    B, T = tokens.shape
    z = plain.embed(tokens, p["table"], enc.scale, lengths) @ p["w_in"]
    v, _ = plain.conv(z[..., :enc.columns], p["taps"], p["taps_bias"], lengths)
    x = v[..., :H * P].reshape(B, T, H, P)
    b, c = (t.reshape(B, T, G, N) for t in np.split(v[..., H * P:], 2, axis=2))
    y, _, _ = plain.scan(x, b, c, z[..., enc.columns:enc.columns + H], -np.exp(p["log_rate"]), p["skip"], p["dt_bias"], lengths,
                         np.zeros((B, H, P, N)))
    emis = y.reshape(B, T, H * P) @ p["w_out"]
    logz = oracle.fwd_bwd(emis, np.asarray(lengths, np.int32), p["trans"], p["dur"], center=False).logz
    K, score = p["dur"].shape[0], 0.0
    for i in range(B):
        start, before = 0, None
        while start < lengths[i]:
            end, c = start + 1, labels[i, start]
            while end < lengths[i] and labels[i, end] == c and end - start < K:
                end += 1
            score += emis[i, start:end, c].sum() + p["dur"][end - start - 1, c]
            score += np.log(np.exp(p["trans"][:, c]).sum()) if before is None else p["trans"][before, c]
            start, before = end, c
    return (np.sum(logz) - score) / B


def test_gradients_of_the_whole_model_match_differences():
    enc, crf = model()
    rng = np.random.default_rng(3)
    tokens, lengths = rng.integers(0, 11, (3, 21)).astype(np.int32), np.array([21, 1, 13])
    labels = np.repeat(rng.integers(0, 3, (3, 3)), 7, axis=1)  # segments of seven: longer than K
    to = lambda v, dt: torch.from_numpy(np.ascontiguousarray(v)).to(dt).to(DEV)  # noqa: E731
    loss, grads = encoder.loss_and_gradients(enc, crf, to(tokens, torch.int32), to(lengths, torch.int32), to(labels, torch.int64))
    p = {k: v.double().cpu().numpy() for k, v in {**enc.params, **crf}.items()}
    assert abs(loss.item() - loss64(enc, p, tokens, lengths, labels)) < 1e-5 * max(1.0, abs(loss.item()))
    assert set(grads) == set(p)
    for k, g in grads.items():
        r, g = rng.standard_normal(p[k].shape), g.double().cpu().numpy()
        at = lambda e: loss64(enc, {**p, k: p[k] + e * r}, tokens, lengths, labels)  # noqa: B023,E731
        want = (at(1e-5) - at(-1e-5)) / 2e-5
        assert abs((g * r).sum() - want) < 5e-5 * np.linalg.norm(g) * np.linalg.norm(r), k


def test_a_stream_follows_the_whole_text():
    enc, _ = model()
    tokens = torch.randint(0, 11, (3, 40), device=DEV, dtype=torch.int32)
    whole, _ = enc.emissions(tokens)
    stream = encoder.Stream(enc, 3)
    stream.seen[1] = -1
    for t in range(40):
        e = stream.step(tokens[:, t].contiguous())
        assert (e[[0, 2]] - whole[[0, 2], t]).abs().max() < 1e-4 * whole.abs().max() and not e[1].any()
    assert stream.seen.tolist() == [40, -1, 40]


def test_training_lowers_the_loss():
    """From the uniform loss downwards, in bfloat16: ten steps on one text."""
    enc, crf = model(torch.bfloat16)
    tokens, lengths, labels = encoder.synthetic(8, 60, 11, 3, 5.0, DEV, seed=4)
    everything = {**enc.params, **crf}
    optimizer = torch.optim.SGD(everything.values(), lr=0.02)
    losses = []
    for _ in range(10):
        loss, grads = encoder.loss_and_gradients(enc, crf, tokens, lengths, labels)
        losses.append(loss.item())
        for k, v in grads.items():
            everything[k].grad = v
        optimizer.step()
    assert np.isfinite(losses).all() and losses[-1] < losses[0]
