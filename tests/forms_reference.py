"""The operators between the QKV projection and the output projection by their definitions, in float64 torch operations, with
the sums of the magnitudes of their terms for error bounds."""
import math

import torch


def attention(q, k, v, *, scale=None, cap=0.0, causal=False, documents=None, prefix=None, slopes=None, grad=None):
    """Outputs and, with grad, gradients, as {name: (value, bound of its fp32 error, bound of bf16 roundings)}; lse: value."""
    q, k, v = q.double(), k.double(), v.double()
    (B, n, h, w), (S, kv) = q.shape, k.shape[1:3]
    G, scale = h // kv, scale or w ** -0.5
    rows = lambda x: x.permute(0, 2, 1, 3).contiguous()                       # [B, heads, rows, w]
    qh, kh, vh = rows(q), rows(k).repeat_interleave(G, 1), rows(v).repeat_interleave(G, 1)
    T = lambda x: x.transpose(-1, -2).contiguous()
    key = torch.arange(S, device=q.device)
    pos = key[S - n:]
    see = torch.ones(B, 1, n, S, dtype=torch.bool, device=q.device)
    if causal:
        see = (key[None] <= pos[:, None])[None, None].expand(B, 1, n, S)
        if prefix is not None:
            see = see | (key[None, None, None] < prefix[:, None, None, None])
    dead_q = dead_k = None
    if documents is not None:
        d = documents.long()
        see = see & (d[:, None, S - n:, None] == d[:, None, None, :]) & (d >= 0)[:, None, None, :]
        dead_q, dead_k = (d[:, S - n:] < 0), (d < 0)
        # padding may hold anything: none of it counts
        qh = torch.where(dead_q[:, None, :, None], 0.0, qh)
        kh = torch.where(dead_k[:, None, :, None], 0.0, kh)
        vh = torch.where(dead_k[:, None, :, None], 0.0, vh)
    x = qh @ T(kh) * scale
    size = qh.abs() @ T(kh.abs()) * scale
    damp = torch.ones_like(x)
    if cap:
        t = torch.tanh(x / cap)
        x, damp = cap * t, 1 - t * t
    if slopes is not None:
        far = slopes.double().view(1, h, 1, 1) * (pos[:, None] - key[None]).abs()
        x, size = x - far, size + far.abs()
    x = torch.where(see, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    # Relative fp32 error of a probability: its score's dot product and distance (16 roundings of its terms' magnitude, for its own
    # and the largest score), the cap's tanh (8 roundings of the cap), the exponential and the sum (16 roundings)
    u = 2.0 ** -24
    rel = u * (16 * (size + size.masked_fill(~see, 0).amax(-1, keepdim=True)) + 16 * cap + 32)
    back = lambda y: y.permute(0, 2, 1, 3)
    shared = lambda y: back(y.reshape(B, kv, G, S, w).sum(2))
    out = p @ vh
    half = 2.0 ** -8
    o_term = p @ vh.abs()
    res = {"out": (back(out), back((p * rel) @ vh.abs() + 16 * u * o_term), back(half * o_term + half * out.abs()))}
    if grad is None:
        return res, lse
    g = rows(grad.double())
    if dead_q is not None:
        g = torch.where(dead_q[:, None, :, None], 0.0, g)
    dp = g @ T(vh)
    delta = (g * out).sum(-1, keepdim=True)
    ds = p * (dp - delta) * damp
    mag = g.abs() @ T(vh.abs())
    dmag = (g.abs() * o_term).sum(-1, keepdim=True)
    # fp32 error of ds: its probability's, and those of dp, delta and damp
    e32 = p * (rel * ((dp - delta).abs() * damp + dmag) + 24 * u * (mag + dmag))
    # roundings to bf16 behind it: ds itself, and the stored output (and the probabilities in it) that delta is taken from
    e16 = half * ds.abs() + p * damp * 2 * half * dmag
    grads = {"dq": (back(ds @ kh) * scale, back((e32 + 16 * u * ds.abs()) @ kh.abs()) * scale, back(e16 @ kh.abs()) * scale),
             "dk": (shared(T(ds) @ qh) * scale, shared(T(e32 + 16 * u * ds.abs()) @ qh.abs()) * scale, shared(T(e16) @ qh.abs()) * scale),
             "dv": (shared(T(p) @ g), shared(T(p * rel + 16 * u * p) @ g.abs()), shared(T(p) @ g.abs()) * half)}
    for name, (value, f32, b16) in grads.items():
        res[name] = (value, f32, b16 + half * value.abs())
    return res, lse


def check(got, want, bf16, name):
    """got within its bounds of the definition."""
    value, f32, b16 = want
    # a probability below fp32's smallest normal number, 2^-126, may become zero; times values below 2^20, over fewer than 2^6
    # of them in a sum that holds nothing larger, that is less than 2^-100
    bound = f32 + (b16 if bf16 else 2.0 ** -23 * value.abs()) + 2.0 ** -100
    off = (got.double() - value).abs()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    worst = (off - bound).max().item()
    assert worst <= 0, f"{name}: {worst:.3e} beyond the bound; largest error {off.max().item():.3e} of {value.abs().max().item():.3e}"


def rotary(x, positions, rotary_width, *, interleaved=False, theta=10000.0, scaling="none", factor=1.0, original_length=0, low_turns=1.0,
           high_turns=32.0, magnitude=1.0, inverse=False):
    """x [batch, seq, heads, width] turned, in float64; positions [batch, seq] or None."""
    x = x.double()
    B, S, _, w = x.shape
    r = rotary_width
    if positions is None:
        positions = torch.arange(S, device=x.device).expand(B, S)
    f = theta ** (-2.0 * torch.arange(r // 2, device=x.device, dtype=torch.float64) / max(r, 1))
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        t = ((original_length * f / (2 * math.pi) - low_turns) / (high_turns - low_turns)).clamp(0, 1)
        f = f * (t + (1 - t) / factor)
    angle = positions.double()[:, :, None, None] * f
    c, s = magnitude * torch.cos(angle), magnitude * torch.sin(angle) * (-1 if inverse else 1)
    i = torch.arange(r // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y
