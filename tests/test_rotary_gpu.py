"""mslt_rotary, mslt_head_norm_rotary and its gradients against the definition in float64: both layouts, part of a head, scaled
frequencies, far positions, odd widths and layouts; and the whole way from the projection through the attention and back.

Bounds.  fp32: an angle is off by 2^-32 of a turn and its conversion, 2^-25 of half a turn, so sine and cosine by 2^-22; a turned
element by 2^-21 of the pair's magnitude with the products' roundings; the norm adds a mean of at most 256 squares and a root,
2^-20 of the value.  bf16 results add half a step, 2^-8 of the value."""
import pytest

from paper_2011_13635_amd import binding
import forms_reference as R

pytestmark = pytest.mark.gpu

FORMS = {
    "half": {}, "interleaved": {"interleaved": True}, "linear": {"scaling": "linear", "factor": 4.0},
    "ramp": {"scaling": "ramp", "factor": 8.0, "original_length": 128, "low_turns": 1.0, "high_turns": 16.0, "magnitude": 1.25},
    "theta": {"theta": 500000.0, "interleaved": True},
}
SHAPES = [
    # B, S, q heads, k heads, width, rotary width
    (1, 1, 1, 1, 2, 2), (1, 1, 12, 12, 64, 64), (2, 37, 4, 2, 64, 32), (3, 50, 5, 3, 80, 80), (1, 129, 16, 4, 128, 128), (2, 9, 3, 1, 256, 128),
    (1, 33, 2, 2, 17, 6), (2, 20, 1, 1, 96, 48), (1, 700, 40, 9, 64, 64), (2, 5, 2, 1, 33, 0), (1, 70, 3, 2, 72, 40), (2, 8, 2, 2, 256, 256),
]


def _inputs(torch, dtype, B, S, hq, hk, w, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    return rand(B, S, hq, w).to(dtype), rand(B, S, hk, w).to(dtype), rand


def _close(got, want, size, steps, bf16, name):
    """within `steps` fp32 roundings of the terms' size, and half a step of bf16"""
    off = (got.double() - want).abs()
    bound = steps * 2.0 ** -24 * size + (2.0 ** -8 if bf16 else 2.0 ** -24) * want.abs()
    assert (off <= bound).all(), f"{name}: {(off - bound).max().item():.3e} beyond the bound, {off.max().item():.3e}"


def _pair_size(x, r, interleaved):
    """largest magnitude of an element's pair, twice"""
    x = x.double().abs()
    y = 2 * x.clone()
    if r:
        a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
        m = 2 * (x[..., a] + x[..., b])
        y[..., a], y[..., b] = m, m
    return y


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_rotary(shape, form, dtype):
    import torch
    dt, kw = getattr(torch, dtype), FORMS[form]
    B, S, hq, hk, w, r = shape
    q, k, rand = _inputs(torch, dt, B, S, hq, hk, w)
    f = binding.rotary_form(r, **kw)
    far = torch.randint(-5, 2_000_000, (B, S), device="cuda", dtype=torch.int32)
    for positions in (None, far):
        for inverse in (False, True):
            got = binding.mslt_rotary(q, k, f, positions=positions, inverse=inverse)
            for x, y in zip((q, k), got):
                _close(y, R.rotary(x, positions, r, inverse=inverse, **kw), 2 * _pair_size(x, r, kw.get("interleaved")), 8, dt == torch.bfloat16, form)
    # in place, queries alone: the same values
    alone, none = binding.mslt_rotary(q.clone(), None, f)
    again = q.clone()
    binding.mslt_rotary(again, None, f, out=(again, None))
    assert none is None and torch.equal(alone, binding.mslt_rotary(q, k, f)[0]) and torch.equal(again, alone)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_head_norm_rotary_and_gradients(shape, form, per_head, dtype):
    import torch
    dt, kw, eps = getattr(torch, dtype), FORMS[form], 1e-5
    bf = dt == torch.bfloat16
    B, S, hq, hk, w, r = shape
    q, k, rand = _inputs(torch, dt, B, S, hq, hk, w, 1)
    gains = [1 + 0.3 * rand(*((h, w) if per_head else (w,))) for h in (hq, hk)]
    grads = [rand(*x.shape).to(dt) for x in (q, k)]
    positions = torch.randint(0, 100_000, (B, S), device="cuda", dtype=torch.int32)
    f = binding.rotary_form(r, **kw)
    got = binding.mslt_head_norm_rotary(q, k, *gains, eps, f, positions=positions)
    d = binding.mslt_head_norm_rotary_backward(q, k, *gains, eps, f, *grads, positions=positions)
    for i, (x, gain, dy, what) in enumerate(zip((q, k), gains, grads, "qk")):
        x, gain = x.double(), gain.double()
        rstd = (x.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
        z = x * rstd * gain
        _close(got[i], R.rotary(z, positions, r, **kw), 2 * _pair_size(z, r, kw.get("interleaved")), 16, bf, "y" + what)
        dz = R.rotary(dy, positions, r, inverse=True, **kw)
        size = 2 * _pair_size(dy, r, kw.get("interleaved"))
        terms = dz * x * rstd
        dims = (0, 1) if per_head else (0, 1, 2)
        # each term carries its turn's and its norm's roundings; a sum of partial sums a few more of the terms' magnitudes
        off = (d["dgain_" + what].double() - terms.sum(dims)).abs()
        assert (off <= 2.0 ** -24 * 40 * (size * (x * rstd).abs()).sum(dims)).all(), f"dgain_{what}: {off.max().item():.3e}"
        mean = (dz * gain * x).mean(-1, keepdim=True)
        want = rstd * (dz * gain - x * rstd ** 2 * mean)
        mag = rstd * (size * gain.abs() + x.abs() * rstd ** 2 * (size * gain.abs() * x.abs()).mean(-1, keepdim=True))
        _close(d["d" + what], want, mag, 32, bf, "d" + what)
    # results over the gradients of the outputs: the same values
    own = [g.clone() for g in grads]
    d2 = binding.mslt_head_norm_rotary_backward(q, k, *gains, eps, f, *own, positions=positions, out=own)
    for name in d:
        assert torch.equal(d[name], d2[name]), name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_layouts(dtype):
    """Parts of a packed projection, heads before tokens, rows off the 16-byte grid: the same values, nothing else written."""
    import torch
    dt = getattr(torch, dtype)
    B, S, hq, hk, w = 2, 21, 4, 2, 64
    q, k, rand = _inputs(torch, dt, B, S, hq, hk, w, 2)
    f = binding.rotary_form(64)
    gains = [1 + 0.3 * rand(w) for _ in range(2)]
    want, wantn = binding.mslt_rotary(q, k, f), binding.mslt_head_norm_rotary(q, k, *gains, 1e-6, f)
    head_major = lambda x: x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)

    def off_grid(x):
        room = torch.full((B, S + 1, x.shape[2], w + 3), 5.0, dtype=dt, device="cuda")
        part = room[:, :S, :, 1:w + 1]
        part.copy_(x)
        return room, part

    for lay in (head_major, lambda x: off_grid(x)[1]):
        for a, b in zip(binding.mslt_rotary(lay(q), lay(k), f), want):
            assert torch.equal(a, b)
        for a, b in zip(binding.mslt_head_norm_rotary(lay(q), lay(k), *gains, 1e-6, f), wantn):
            assert (a.double() - b.double()).abs().max() <= 2.0 ** (-6 if dt == torch.bfloat16 else -20)     # (another order of the mean's sum)
    room, part = off_grid(torch.zeros_like(q))
    binding.mslt_rotary(q, k, f, out=(part, torch.empty_like(k)))
    assert torch.equal(part, want[0])
    part.fill_(5.0)
    assert (room == 5).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_offsets_beyond_32_bits(dtype):
    import torch
    dt = getattr(torch, dtype)
    B, S, hq, hk, w = 2, 21, 4, 2, 64
    q, k, rand = _inputs(torch, dt, B, S, hq, hk, w, 2)
    f = binding.rotary_form(64)
    room = torch.empty((1 << 32) + 4 * (1 << 30) + S * (1 << 20), dtype=dt, device="cuda")

    def spread(x, at):
        y = room.as_strided(x.shape, (1 << 32, 1 << 20, 1 << 30, 1), at)
        y.copy_(x)
        return y

    gains = [1 + 0.3 * rand(w) for _ in range(2)]
    q2, k2 = spread(q, 0), spread(k, 64)
    for got, want in zip(binding.mslt_rotary(q2, k2, f), binding.mslt_rotary(q, k, f)):
        assert torch.equal(got, want)
    a, b = (binding.mslt_head_norm_rotary_backward(*x, *gains, 1e-6, f, *x) for x in ((q, k), (q2, k2)))
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_padding_rows_of_zeros_and_large_values():
    import torch
    x = torch.zeros(1, 3, 2, 64, device="cuda")
    x[0, 1] = 1e18           # its squares pass fp32's range only in the sum: 64e36 is below 3.4e38
    gains = [torch.ones(64, device="cuda")] * 2
    f = binding.rotary_form(0)
    y, _ = binding.mslt_head_norm_rotary(x, x, *gains, 1e-6, f)
    assert (y[0, 0] == 0).all() and ((y[0, 1] - 1).abs() < 1e-6).all()
    d = binding.mslt_head_norm_rotary_backward(x, x, *gains, 1e-6, f, torch.ones_like(x), torch.ones_like(x))
    assert all(torch.isfinite(t).all() for t in d.values())
    assert ((d["dq"][0, 0] - 1000).abs() < 1e-2).all()      # rows of zeros: 1 / sqrt(eps)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("heads", [(4, 4, 64), (6, 2, 128)])
def test_from_the_projection_through_the_attention_and_back(heads, dtype):
    """As a layer uses them: norm and rotation of a packed projection's queries and keys, attention over packed documents, and
    back, with every operator's gradient handed to the next; each against the definition on the operands it got.  Captured
    into a graph and replayed between eager calls: the same values."""
    import torch
    dt = getattr(torch, dtype)
    bf = dt == torch.bfloat16
    (h, kv, w), B, S, eps = heads, 2, 140, 1e-6
    g = torch.Generator(device="cuda").manual_seed(11)
    qkv = torch.randn((B, S, (h + 2 * kv) * w), generator=g, device="cuda").to(dt)
    part = lambda x, at, n: x[..., at * w:(at + n) * w].view(B, S, n, w)
    q, k, v = part(qkv, 0, h), part(qkv, h, kv), part(qkv, h + kv, kv)
    gains = [1 + 0.2 * torch.randn(w, generator=g, device="cuda") for _ in range(2)]
    go = torch.randn((B, S, h, w), generator=g, device="cuda").to(dt)
    docs = torch.zeros(B, S, dtype=torch.int32, device="cuda")
    docs[:, 60:] = 1
    docs[1, 120:] = -1
    positions = torch.where(docs == 1, torch.arange(S, device="cuda") - 60, torch.arange(S, device="cuda")).to(torch.int32)
    rot, form = binding.rotary_form(w // 2, interleaved=True), binding.attention_form(cap=20.0)
    dqkv = torch.zeros_like(qkv)

    def step():
        qn, kn = binding.mslt_head_norm_rotary(q, k, *gains, eps, rot, positions=positions)
        f = binding.mslt_attention(qn, kn, v, form, documents=docs)
        d = binding.mslt_attention_backward(qn, kn, v, f["out"], f["lse"], go, form, documents=docs, grads=(part(dqkv, 0, h), part(dqkv, h, kv), part(dqkv, h + kv, kv)))
        dqn, dkn = d["dq"].clone(), d["dk"].clone()
        n = binding.mslt_head_norm_rotary_backward(q, k, *gains, eps, rot, d["dq"], d["dk"], positions=positions, out=(d["dq"], d["dk"]))
        return {"qn": qn, "kn": kn, "out": f["out"], "dqn": dqn, "dkn": dkn, "dgain_q": n["dgain_q"], "dgain_k": n["dgain_k"], "dqkv": dqkv}

    got = {name: t.clone() for name, t in step().items()}
    want, _ = R.attention(got["qn"], got["kn"], v, cap=20.0, documents=docs, grad=go)
    for name, mine in (("out", got["out"]), ("dq", got["dqn"]), ("dk", got["dkn"]), ("dv", part(got["dqkv"], h + kv, kv))):
        R.check(mine, want[name], bf, name)
    for x, gain, dy, dx, dg, y in ((q, gains[0], "dqn", part(got["dqkv"], 0, h), "dgain_q", "qn"), (k, gains[1], "dkn", part(got["dqkv"], h, kv), "dgain_k", "kn")):
        x, gain = x.double(), gain.double()
        rstd = (x.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
        z = x * rstd * gain
        _close(got[y], R.rotary(z, positions, w // 2, interleaved=True), 2 * _pair_size(z, w // 2, True), 16, bf, y)
        dz = R.rotary(got[dy], positions, w // 2, interleaved=True, inverse=True)
        size = 2 * _pair_size(got[dy], w // 2, True)
        terms = dz * x * rstd
        assert ((got[dg].double() - terms.sum((0, 1, 2))).abs() <= 2.0 ** -24 * 40 * (size * (x * rstd).abs()).sum((0, 1, 2))).all(), dg
        dx_want = rstd * (dz * gain - x * rstd ** 2 * (dz * gain * x).mean(-1, keepdim=True))
        mag = rstd * (size * gain.abs() + x.abs() * rstd ** 2 * (size * gain.abs() * x.abs()).mean(-1, keepdim=True))
        _close(dx, dx_want, mag, 32, bf, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(3):
        for t in captured.values():
            t.fill_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        for name, t in captured.items():
            assert torch.equal(t, got[name]), name
        eager = step()
        torch.cuda.synchronize()
        for name, t in eager.items():
            assert torch.equal(t, got[name]), name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 2, 1, 64), (1, 7, 3, 2, 64), (3, 5, 4, 4, 128), (1, 4099, 12, 4, 64), (2, 3, 2, 2, 33)], ids=lambda s: "x".join(map(str, s)))
def test_norm_without_eps(shape, per_head, dtype):
    """eps = 0 is allowed; what a workgroup works on behind the last token, rows of zeros whose norm is none, adds nothing to the gains'
    gradients.  The bounds are those of test_head_norm_rotary_and_gradients."""
    import torch
    dt = getattr(torch, dtype)
    B, S, hq, hk, w = shape
    q, k, rand = _inputs(torch, dt, B, S, hq, hk, w, 3)
    gains = [1 + 0.3 * rand(*((h, w) if per_head else (w,))) for h in (hq, hk)]
    grads = [rand(*x.shape).to(dt) for x in (q, k)]
    f = binding.rotary_form(32)
    got = binding.mslt_head_norm_rotary(q, k, *gains, 0.0, f)
    d = binding.mslt_head_norm_rotary_backward(q, k, *gains, 0.0, f, *grads)
    for i, (x, gain, dy, what) in enumerate(zip((q, k), gains, grads, "qk")):
        x, gain = x.double(), gain.double()
        rstd = x.pow(2).mean(-1, keepdim=True).rsqrt()
        z = x * rstd * gain
        _close(got[i], R.rotary(z, None, 32), 2 * _pair_size(z, 32, False), 16, dt == torch.bfloat16, "y" + what)
        dz = R.rotary(dy, None, 32, inverse=True)
        size, dims = 2 * _pair_size(dy, 32, False), (0, 1) if per_head else (0, 1, 2)
        off = (d["dgain_" + what].double() - (dz * x * rstd).sum(dims)).abs()
        assert (off <= 2.0 ** -24 * 40 * (size * (x * rstd).abs()).sum(dims)).all(), f"dgain_{what}: {off.max().item():.3e}"
        want = rstd * (dz * gain - x * rstd ** 2 * (dz * gain * x).mean(-1, keepdim=True))
        mag = rstd * (size * gain.abs() + x.abs() * rstd ** 2 * (size * gain.abs() * x.abs()).mean(-1, keepdim=True))
        _close(d["d" + what], want, mag, 32, dt == torch.bfloat16, "d" + what)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads", [(2, 1), (3, 2), (5, 2), (11, 0)])
def test_workgroups_that_no_whole_wavefronts_fill(heads, interleaved, dtype):
    """3, 5, 7 and 11 heads of 64 leave lanes of a workgroup's last wavefront without a token: these look nothing up."""
    import torch
    dt, (hq, hk) = getattr(torch, dtype), heads
    q, k, rand = _inputs(torch, dt, 2, 83, hq, max(hk, 1), 64, 5)
    f = binding.rotary_form(64, interleaved=interleaved)
    for x, y in zip((q, k), binding.mslt_rotary(q, k if hk else None, f)[:2 if hk else 1]):
        _close(y, R.rotary(x, None, 64, interleaved=interleaved), 2 * _pair_size(x, 64, interleaved), 8, dt == torch.bfloat16, "y")
