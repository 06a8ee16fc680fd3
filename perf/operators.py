"""The operators between a layer's QKV projection and its output projection: what a case is, its inputs, one pass.

Three operators, used one after the other: rotary positions (`mslt_rotary`), the norm of queries and keys for each head
with the rotation in the same pass (`mslt_head_norm_rotary`), and attention with a score cap, a distance bias, a document
mask and a prefix mask (`mslt_attention`).  Queries, keys and values are views of one packed projection [batch, seq,
(heads + 2 kv_heads) * width], as a layer's QKV product leaves it; a single query over a cache comes as its own tensor.

`run` computes the plain form in fp32 from elementary operations (angles in fp64: they lose their digits at far positions).
"""
import math
import random

import numpy as np
import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-6
_THETA = 10000.0


def _rotary(name, dtype, batch, seq, heads, kv_heads, width, rotary, interleaved=False, scaling="none", far=0, inverse=False):
    """Rotary positions of queries and keys; far: position of the first token."""
    return {"name": name, "op": "rotary", "dtype": dtype, "batch": batch, "seq": seq, "heads": heads, "kv_heads": kv_heads, "width": width,
            "rotary": rotary, "interleaved": interleaved, "scaling": scaling, "far": far, "inverse": inverse}


def _norm(name, dtype, batch, seq, heads, kv_heads, width, rotary, interleaved=False, scaling="none", per_head=False, backward=False):
    """Norm of each head of queries and keys with the rotation, and its gradients."""
    return {"name": name, "op": "norm", "dtype": dtype, "batch": batch, "seq": seq, "heads": heads, "kv_heads": kv_heads, "width": width,
            "rotary": rotary, "interleaved": interleaved, "scaling": scaling, "per_head": per_head, "backward": backward, "far": 0}


def _attention(name, dtype, batch, queries, seq, heads, kv_heads, width, cap=0.0, mask="full", documents=0, padding=0.0, slopes=False,
               backward=False):
    """queries of the last positions over seq keys; documents: mean length of those packed into a row (twice seq or more: one), 0: none; padding:
    share of a row behind its last document; mask: full, causal or prefix."""
    return {"name": name, "op": "attention", "dtype": dtype, "batch": batch, "queries": queries, "seq": seq, "heads": heads,
            "kv_heads": kv_heads, "width": width, "cap": cap, "mask": mask, "documents": documents, "padding": padding,
            "slopes": slopes, "backward": backward}


def listed():
    return [
        # one token far into a long text: a call's latency
        _rotary("rotary_one_token", "bf16", 1, 1, 12, 12, 64, 64, far=100_003),
        # gradient of the rotation of half a head, fp32 mode, a batch padded to its longest sequence
        _rotary("rotary_back_fp32_27x203", "fp32", 27, 203, 12, 12, 64, 32, interleaved=True, inverse=True),
        # grouped heads over long contexts whose positions are scaled: pure bandwidth
        _rotary("rotary_scaled_4x16384", "bf16", 4, 16384, 16, 4, 128, 128, scaling="ramp"),
        # a small fp32 step, forward and backward, with which bf16 training is compared
        _norm("norm_fp32_8x128", "fp32", 8, 128, 12, 12, 64, 64, backward=True),
        # one long odd sequence, gains for each head, interleaved pairs in half the head
        _norm("norm_1x4099", "bf16", 1, 4099, 16, 4, 128, 64, interleaved=True, scaling="linear", per_head=True),
        # a layer of the largest step, forward and backward
        _norm("norm_train_32x512", "bf16", 32, 512, 16, 16, 64, 64, backward=True),
        # one new token for each of eight sequences over their kept keys, grouped heads, capped scores, some rows shorter
        _attention("attention_one_query_8x8191", "bf16", 8, 1, 8191, 16, 4, 128, cap=30.0, mask="causal", documents=16382, padding=0.1),
        # a small fp32 training layer at an odd length with packed documents and a distance bias
        _attention("attention_fp32_3x203", "fp32", 3, 203, 203, 12, 12, 64, documents=60, padding=0.1, slopes=True, backward=True),
        # a layer of the headline step: a padded batch of short sequences
        _attention("attention_train_64x128", "bf16", 64, 128, 128, 16, 16, 64, documents=256, padding=0.2, backward=True),
        # a layer of the largest step, short documents packed into rows, capped scores
        _attention("attention_packed_32x512", "bf16", 32, 512, 512, 16, 16, 64, cap=50.0, documents=170, padding=0.05, backward=True),
        # prefix language modelling over one long sequence, grouped heads, a distance bias
        _attention("attention_prefix_1x8192", "bf16", 1, 8192, 8192, 16, 4, 128, mask="prefix", slopes=True, backward=True),
        # scores of a long text, everything sees everything, forward only
        _attention("attention_long_1x16384", "bf16", 1, 16384, 16384, 12, 12, 64, cap=50.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; never more than the largest of them costs."""
    op = rng.choices(["rotary", "norm", "attention"], [2, 3, 6])[0]
    dtype = rng.choices(["bf16", "fp32"], [3, 1])[0]
    width = rng.choice([32, 64, 64, 64, 80, 96, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 6, 8, 12, 16])
    heads = kv_heads * rng.choice([1, 1, 1, 2, 3, 4])
    if op != "attention":
        tokens = _log_int(rng, 1, 65536 if dtype == "bf16" else 16384)
        batch = min(tokens, _log_int(rng, 1, 64))
        seq = max(1, tokens // batch)
        rotary = rng.choice([width, width, width // 2])
        layout, scaling = rng.random() < 0.4, rng.choice(["none", "none", "linear", "ramp"])
        if op == "rotary":
            far = rng.choice([0, 0, _log_int(rng, 1, 1_000_000)])
            case = _rotary("", dtype, batch, seq, heads, kv_heads, width, rotary, layout, scaling, far, rng.random() < 0.4)
        else:
            case = _norm("", dtype, batch, seq, heads, kv_heads, width, rotary, layout, scaling, rng.random() < 0.3, rng.random() < 0.6)
        # bytes of a pass: at most those of rotary_scaled_4x16384
        most = 4 * 16384 * 20 * 128 * 2 * 2 // ((5 if case.get("backward") else 2) * (heads + kv_heads) * width * (2 if dtype == "bf16" else 4))
        case["seq"] = min(seq, most)
        case["batch"] = max(1, min(batch, most // case["seq"]))
    else:
        cap = rng.choice([0.0, 0.0, 20.0, 50.0])
        mask = rng.choice(["full", "causal", "prefix"])
        documents = 0 if mask == "prefix" else rng.choice([0, 1, 1])
        padding, slopes = rng.choice([0.0, 0.1, 0.3]) if documents else 0.0, rng.random() < 0.4
        one = rng.random() < 0.25
        seq = _log_int(rng, 1, 16384 if dtype == "bf16" else 4096)
        queries = rng.randint(1, min(seq, 4)) if one else seq
        backward = not one and rng.random() < 0.6
        # products of a pass: at most those of attention_prefix_1x8192, and the plain form's scores at most 3.2e9 (1.07e9 with
        # gradients); in fp32 mode a sixteenth
        most = min(6.9e10 / width, 1.07e9) if backward else min(2.06e11 / width, 3.2e9)
        most = int(most if dtype == "bf16" else most / 16)
        while queries * seq * heads > most:
            if heads > 4:
                kv_heads, heads = max(1, kv_heads // 2), max(1, kv_heads // 2) * (heads // kv_heads)
            else:
                seq = seq * 3 // 4
                queries = min(queries, seq) if one else seq
        batch = max(1, min(_log_int(rng, 1, 64), most // (queries * seq * heads), 8 * 8192 * 1024 // (seq * kv_heads * width) + 1))
        size = 6 * (queries * heads + seq * kv_heads) * width * 4 if backward else 2 * (queries * heads + seq * kv_heads) * width * 4
        batch = max(1, min(batch, 500_000_000 // size))
        documents = (2 * seq if rng.random() < (0.7 if one else 0.3) else _log_int(rng, 16, max(17, seq))) if documents else 0
        case = _attention("", dtype, batch, queries, seq, heads, kv_heads, width, cap, mask, documents, padding, slopes, backward)
    del case["name"]
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _document_lengths(case):
    """Lengths of the documents of each row, by the case alone: the work does not depend on the seed."""
    rng = random.Random("%d %d %d %g" % (case["batch"], case["seq"], case["documents"], case["padding"]))
    rows = []
    for _ in range(case["batch"]):
        left = case["seq"] - int(round(case["seq"] * case["padding"] * rng.random()))
        lengths = []
        while left > 0:
            n = min(left, max(1, int(case["documents"] * rng.uniform(0.5, 1.5))))
            lengths.append(n)
            left -= n
        rows.append(lengths)
    return rows


def _prefixes(case):
    rng = random.Random("%d %d" % (case["batch"], case["seq"]))
    return [int(case["seq"] * rng.uniform(0.05, 0.4)) for _ in range(case["batch"])]


def prepare(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    dtype, B, S, h, kv, w = _DTYPE[case["dtype"]], case["batch"], case["seq"], case["heads"], case["kv_heads"], case["width"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=device, dtype=torch.float32)

    state = {"case": case}
    packed = normal(B, S, (h + 2 * kv) * w)
    if case["op"] == "attention":   # sharper than chance, as trained scores are; capped ones reach into the cap
        packed[..., :(h + kv) * w] *= 1.5 if case["cap"] == 0 else 2.0
    packed = packed.to(dtype)
    state["q"] = packed[..., :h * w].view(B, S, h, w)
    state["k"] = packed[..., h * w:(h + kv) * w].view(B, S, kv, w)
    state["v"] = packed[..., (h + kv) * w:].view(B, S, kv, w)
    if case["op"] != "attention":
        pos = torch.arange(S, device=device, dtype=torch.int32) + case["far"]
        state["positions"] = pos.expand(B, S).contiguous()
        if own:
            from paper_2011_13635_amd import binding
            state["form"] = binding.rotary_form(case["rotary"], interleaved=case["interleaved"], theta=_THETA, scaling=case["scaling"],
                                                factor=8.0, original_length=2048, low_turns=1.0, high_turns=32.0,
                                                magnitude=1.2 if case["scaling"] == "ramp" else 1.0)
        if case["op"] == "norm":
            state["gain_q"] = 1.0 + 0.2 * normal(*((h, w) if case["per_head"] else (w,)))
            state["gain_k"] = 1.0 + 0.2 * normal(*((kv, w) if case["per_head"] else (w,)))
            if case["backward"]:
                state["dq"] = normal(B, S, h, w).to(dtype)
                state["dk"] = normal(B, S, kv, w).to(dtype)
        return state
    if case["queries"] < S:
        state["q"] = state["q"][:, S - case["queries"]:].contiguous()
    if case["backward"]:
        state["dout"] = normal(B, case["queries"], h, w).to(dtype)
    state["documents"] = state["prefix"] = state["slopes"] = None
    if case["documents"]:
        rng, ids = random.Random(seed), np.full((B, S), -1, dtype=np.int32)
        rows = _document_lengths(case)
        rng.shuffle(rows)
        for b, lengths in enumerate(rows):
            n = sum(lengths)
            if case["queries"] == S:
                rng.shuffle(lengths)
            lo = S - n if case["queries"] < S else 0      # a cache is padded in front, so that the new token is the last
            ids[b, lo:lo + n] = np.repeat(np.arange(len(lengths), dtype=np.int32), lengths)
        state["documents"] = torch.from_numpy(ids).to(device)
    if case["mask"] == "prefix":
        state["prefix"] = torch.tensor(_prefixes(case), dtype=torch.int32, device=device)[torch.randperm(B, generator=g, device=device)]
    if case["slopes"]:
        state["slopes"] = torch.exp2(-8.0 * (torch.arange(h, device=device, dtype=torch.float32) + 1) / h) * (1.0 + 0.1 * normal(h))
    if own:
        from paper_2011_13635_amd import binding
        state["form"] = binding.attention_form(cap=case["cap"], causal=case["mask"] != "full")
    return state


# ---- one pass -------------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    return {"rotary": _run_rotary, "norm": _run_norm, "attention": _run_attention}[case["op"]](case, state)


def _frequencies(case, device, dtype=torch.float64):
    r = case["rotary"]
    f = _THETA ** (-torch.arange(0, r, 2, device=device, dtype=dtype) / r)
    if case["scaling"] == "linear":
        f = f / 8.0
    if case["scaling"] == "ramp":
        t = ((f * (2048 / (2 * math.pi)) - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * (t + (1.0 - t) / 8.0)
    return f


def _turn(x, case, cos, sin):
    """The rotation of x [B, S, heads, width] by angles [B, S, 1, rotary / 2]."""
    r = case["rotary"]
    head, tail = x[..., :r], x[..., r:]
    a, b = (head[..., 0::2], head[..., 1::2]) if case["interleaved"] else (head[..., :r // 2], head[..., r // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    head = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((head, tail), -1)


def _angles(case, state):
    angle = state["positions"].to(torch.float64)[:, :, None, None] * _frequencies(case, state["positions"].device)
    m = 1.2 if case["scaling"] == "ramp" else 1.0
    return (m * torch.cos(angle)).float(), (m * torch.sin(angle)).float()


def _run_rotary(case, state):
    q, k = state["q"], state["k"]
    if own:
        from paper_2011_13635_amd import binding
        return binding.mslt_rotary(q, k, state["form"], positions=state["positions"], inverse=case["inverse"])
    cos, sin = _angles(case, state)
    if case["inverse"]:
        sin = -sin
    return _turn(q.float(), case, cos, sin).to(q.dtype), _turn(k.float(), case, cos, sin).to(k.dtype)


def _run_norm(case, state):
    q, k = state["q"], state["k"]
    if own:
        from paper_2011_13635_amd import binding
        args = (q, k, state["gain_q"], state["gain_k"], _EPS, state["form"])
        y = binding.mslt_head_norm_rotary(*args, positions=state["positions"])
        if not case["backward"]:
            return y
        d = binding.mslt_head_norm_rotary_backward(*args, state["dq"], state["dk"], positions=state["positions"])
        return *y, d["dq"], d["dk"], d["dgain_q"], d["dgain_k"]
    cos, sin = _angles(case, state)

    def forward(x, gain):
        x = x.float()
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
        return _turn(x * rstd * gain, case, cos, sin)

    def backward(x, gain, dy):
        x = x.float()
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
        dz, xhat = _turn(dy.float(), case, cos, -sin), x * rstd
        dgain = (dz * xhat).sum((0, 1) if case["per_head"] else (0, 1, 2))
        dg = dz * gain
        return (rstd * (dg - xhat * (dg * xhat).mean(-1, keepdim=True))).to(dy.dtype), dgain

    y = forward(q, state["gain_q"]).to(q.dtype), forward(k, state["gain_k"]).to(k.dtype)
    if not case["backward"]:
        return y
    dq, dgq = backward(q, state["gain_q"], state["dq"])
    dk, dgk = backward(k, state["gain_k"], state["dk"])
    return *y, dq, dk, dgq, dgk


def _run_attention(case, state):
    q, k, v = state["q"], state["k"], state["v"]
    if own:
        from paper_2011_13635_amd import binding
        masks = {"documents": state["documents"], "prefix": state["prefix"], "slopes": state["slopes"]}
        f = binding.mslt_attention(q, k, v, state["form"], **masks)
        if not case["backward"]:
            return f["out"], f["lse"]
        d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], state["dout"], state["form"], **masks)
        return f["out"], f["lse"], d["dq"], d["dk"], d["dv"]
    B, n, h, w = q.shape
    S, kv = k.shape[1], k.shape[2]
    group, scale = h // kv, 1.0 / math.sqrt(w)
    # [B, kv, group, rows, width]
    qf = q.float().view(B, n, kv, group, w).permute(0, 2, 3, 1, 4).contiguous()
    kf = k.float().permute(0, 2, 1, 3)[:, :, None].expand(B, kv, group, S, w).contiguous()
    vf = v.float().permute(0, 2, 1, 3)[:, :, None].expand(B, kv, group, S, w).contiguous()
    s = torch.matmul(qf, kf.transpose(-1, -2).contiguous()) * scale
    damp = None
    if case["cap"]:
        t = torch.tanh(s / case["cap"])
        s = case["cap"] * t
        damp = 1.0 - t * t if case["backward"] else None
    key = torch.arange(S, device=q.device)
    pos = key[S - n:]
    if state["slopes"] is not None:
        s = s - state["slopes"].view(kv, group, 1, 1) * (pos[:, None] - key).abs()
    seen = torch.ones(1, 1, 1, n, S, dtype=torch.bool, device=q.device)
    if case["mask"] != "full":
        seen = (key <= pos[:, None])[None, None, None]
    if state["prefix"] is not None:
        seen = seen | (key < state["prefix"].view(B, 1, 1, 1, 1))
    if state["documents"] is not None:
        ids = state["documents"]
        seen = seen & ((ids[:, None, None, S - n:, None] == ids[:, None, None, None, :]) & (ids >= 0)[:, None, None, None, :])
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    out = torch.matmul(p, vf)
    lse = (top + torch.log(total)).view(B, h, n)

    def rows(x):
        return x.permute(0, 3, 1, 2, 4).reshape(B, n, h, w).to(q.dtype)

    if not case["backward"]:
        return rows(out), lse
    go = state["dout"].float().view(B, n, kv, group, w).permute(0, 2, 3, 1, 4).contiguous()
    dp = torch.matmul(go, vf.transpose(-1, -2).contiguous())
    ds = p * (dp - (go * out).sum(-1, keepdim=True)) * scale
    if damp is not None:
        ds = ds * damp
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), qf).sum(2).permute(0, 2, 1, 3)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), go).sum(2).permute(0, 2, 1, 3)
    return rows(out), lse, rows(torch.matmul(ds, kf)), dk.to(k.dtype).contiguous(), dv.to(v.dtype).contiguous()


# ---- from the definition, in 64 bits ----------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, state)
    B, S, r, w = case["batch"], case["seq"], case["rotary"], case["width"]
    device = state["q"].device
    sign, m = (-1.0 if case.get("inverse") else 1.0), (1.2 if case["scaling"] == "ramp" else 1.0)
    # the rotation of a head as complex numbers: pair i turns by exp(sqrt(-1) * position * frequency_i)
    i = torch.arange(r // 2, device=device, dtype=torch.float64)
    freq = torch.exp(i * (-2.0 / r * math.log(_THETA)))
    if case["scaling"] == "linear":
        freq = freq * 0.125
    elif case["scaling"] == "ramp":
        share = torch.clamp((2048.0 * freq / math.tau - 1.0) / (32.0 - 1.0), min=0.0, max=1.0)
        freq = share * freq + (1.0 - share) * freq / 8.0
    phase = state["positions"].double().unsqueeze(-1) * freq
    unit = torch.polar(torch.full_like(phase, m), phase)
    first = (2 * i if case["interleaved"] else i).long()
    second = (2 * i + 1 if case["interleaved"] else i + r // 2).long()

    def turned(x, conj):
        z = torch.complex(x[..., first], x[..., second]) * (unit.conj() if conj else unit).unsqueeze(2)
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    if case["op"] == "rotary":
        return turned(state["q"].double(), sign < 0), turned(state["k"].double(), sign < 0)
    outs, grads, gains = [], [], []
    for x, gain, dy in ((state["q"], state["gain_q"], state.get("dq")), (state["k"], state["gain_k"], state.get("dk"))):
        x, gain = x.double(), gain.double()
        length = torch.sqrt(x.pow(2).sum(-1, keepdim=True) / w + _EPS)
        outs.append(turned(x / length * gain, False))
        if dy is None:
            continue
        dz = turned(dy.double(), True)
        part = dz * x / length
        gains.append(part.reshape(B * S, -1, w).sum(0) if case["per_head"] else part.reshape(-1, w).sum(0))
        weighted = dz * gain
        grads.append(weighted / length - x * (weighted * x).sum(-1, keepdim=True) / (w * length.pow(3)))
    return (*outs, *grads, *gains)


def _exact_attention(case, state):
    q, k, v = state["q"], state["k"], state["v"]
    B, n, h, w = q.shape
    S, group = k.shape[1], h // k.shape[2]
    f64 = {"dtype": torch.float64, "device": q.device}
    out, lse = torch.zeros(B, n, h, w, **f64), torch.zeros(B, h, n, **f64)
    dq, dk, dv = torch.zeros(q.shape, **f64), torch.zeros(k.shape, **f64), torch.zeros(v.shape, **f64)
    at = torch.arange(S, device=q.device)
    far = (at[S - n:].unsqueeze(1) - at).abs().double()
    for b in range(B):
        hidden = torch.zeros(n, S, dtype=torch.bool, device=q.device)
        if case["mask"] != "full":
            hidden = at.unsqueeze(0) > at[S - n:].unsqueeze(1)
        if state["prefix"] is not None:
            hidden = hidden & (at >= state["prefix"][b]).unsqueeze(0)
        if state["documents"] is not None:
            d = state["documents"][b]
            hidden = hidden | (d[S - n:].unsqueeze(1) != d.unsqueeze(0)) | (d < 0).unsqueeze(0)
        some = ~hidden.all(1)
        for j in range(h):
            qj, kj, vj = q[b, :, j].double(), k[b, :, j // group].double(), v[b, :, j // group].double()
            a = qj @ kj.T.contiguous() / math.sqrt(w)
            slope = None
            if case["cap"]:
                a = torch.tanh(a / case["cap"]) * case["cap"]
                slope = 1.0 - (a / case["cap"]) ** 2
            if state["slopes"] is not None:
                a = a - far * state["slopes"][j].double()
            a.masked_fill_(hidden, -math.inf)
            lse[b, j] = torch.logsumexp(a, 1)
            a = torch.exp(a - torch.where(some, lse[b, j], 0.0).unsqueeze(1))
            out[b, :, j] = a @ vj
            if case["backward"]:
                gj = state["dout"][b, :, j].double()
                dv[b, :, j // group] += a.T.contiguous() @ gj
                dp = gj @ vj.T.contiguous()
                da = a * (dp - (a * dp).sum(1, keepdim=True))
                if slope is not None:
                    da = da * slope
                dq[b, :, j] = da @ kj / math.sqrt(w)
                dk[b, :, j // group] += da.T.contiguous() @ qj / math.sqrt(w)
    return (out, lse, dq, dk, dv) if case["backward"] else (out, lse)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
def _pairs(case):
    """Query-key pairs that see each other, and keys that any query may see, over the batch."""
    B, n, S = case["batch"], case["queries"], case["seq"]
    if case["mask"] == "prefix":
        pos = np.arange(S - n, S, dtype=np.int64) + 1
        return int(sum(np.maximum(pos, p).sum() for p in _prefixes(case))), B * S
    rows = _document_lengths(case) if case["documents"] else [[S]] * B
    pairs = keys = 0
    for lengths in rows:
        if n < S:       # the last queries; one document holds them but for a case's rare short last one
            last = lengths[-1]
            m = min(n, last)
            pairs += sum(last - i for i in range(m)) if case["mask"] == "causal" else m * last
            keys += last
        else:
            pairs += sum(m * (m + 1) // 2 if case["mask"] == "causal" else m * m for m in lengths)
            keys += sum(lengths)
    return pairs, keys


def work(case):
    e, w, h, kv = (2 if case["dtype"] == "bf16" else 4), case["width"], case["heads"], case["kv_heads"]
    if case["op"] != "attention":
        x = case["batch"] * case["seq"] * (h + kv) * w
        passes = 5 if case.get("backward") else 2      # forward reads and writes x; backward reads x and the gradient, writes one
        return {"bytes": passes * x * e, "flops": (6 if case["op"] == "rotary" else 30 if case["backward"] else 10) * x}
    pairs, keys = _pairs(case)
    rows = case["batch"] * case["queries"]
    q, k = rows * h * w * e, keys * kv * w * e
    if not case["backward"]:
        return {"bytes": 2 * q + 2 * k + 4 * rows * h, "flops": 4 * pairs * h * w}
    # forward, then backward: q, k, v, out and its gradient in; three gradients out
    return {"bytes": 6 * q + 6 * k + 8 * rows * h, "flops": 14 * pairs * h * w}
