"""mslt_attention and its gradients against the definition in float64: caps, distance biases, document and prefix masks, grouped
heads, few queries over many keys, odd lengths and widths, layouts, padding that holds NaN, streams, graphs.

Bounds are derived in forms_reference: fp32 roundings of every term, and in bf16 mode half a step (2^-8 of the value) for the
probabilities, for dS, for the stored output that delta is taken from, and for each result."""
import pytest

from paper_2011_13635_amd import binding
import forms_reference as R

pytestmark = pytest.mark.gpu


def _documents(torch, B, S, kind, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "packed":       # several in a row, padding behind them; the last sequence is padding alone
        ids = torch.sort(torch.randint(0, 4, (B, S), generator=g), 1).values
        ids[:, S - S // 5:] = -1
        if B > 1:
            ids[-1] = -1
    elif kind == "mixed":      # in no order, entries far apart, padding in between
        ids = torch.randint(0, 3, (B, S), generator=g) * 1_000_003
        ids[torch.rand(B, S, generator=g) < 0.2] = -7
    else:                      # front: padded in front, as a cache is
        ids = torch.zeros(B, S, dtype=torch.long)
        ids[:, :S // 3] = -1
    return ids.to(torch.int32).cuda()


def _case(torch, dtype, B, n, S, h, kv, w, *, cap=0.0, causal=False, documents=None, prefix=False, slopes=False, backward=True, seed=0,
          sharp=1.5, nan_padding=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    qkv = torch.randn((B, S, (h + 2 * kv) * w), generator=g, device="cuda")
    qkv[..., :(h + kv) * w] *= sharp
    qkv = qkv.to(dtype)
    q = qkv[:, S - n:, :h * w].view(B, n, h, w)
    k = qkv[..., h * w:(h + kv) * w].view(B, S, kv, w)
    v = qkv[..., (h + kv) * w:].view(B, S, kv, w)
    grad = rand(B, n, h, w)
    masks = {"documents": _documents(torch, B, S, documents, seed) if documents else None,
             "prefix": torch.randint(-2, S + 3, (B,), generator=g, device="cuda", dtype=torch.int32) if prefix else None,
             "slopes": (torch.rand(h, generator=g, device="cuda") - 0.2) * 16.0 / S if slopes else None}
    if nan_padding:
        dead = masks["documents"] < 0
        qkv[dead] = float("nan")
        grad[dead[:, S - n:]] = float("inf")
    f = binding.mslt_attention(q, k, v, binding.attention_form(cap=cap, causal=causal), **masks)
    want, lse = R.attention(q, k, v, cap=cap, causal=causal, grad=grad if backward else None, **masks)
    got = dict(f)
    if backward:
        got.update(binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], grad, binding.attention_form(cap=cap, causal=causal), **masks))
    torch.cuda.synchronize()
    for name, w3 in want.items():
        R.check(got[name], w3, dtype == torch.bfloat16, name)
    empty = torch.isinf(lse)
    assert torch.equal(empty, torch.isinf(f["lse"])) and (f["lse"][empty] < 0).all()
    # score terms add up to at most a few hundred here: 2^-12 is 16 roundings of one of 2^8
    assert ((f["lse"].double() - lse)[~empty].abs() <= 2.0 ** -12).all()
    return got


SHAPES = [
    # B, queries, keys, heads, kv_heads, width
    (1, 1, 1, 1, 1, 8), (2, 1, 1, 4, 2, 64), (1, 2, 3, 2, 1, 64), (2, 31, 31, 2, 2, 32), (1, 33, 33, 3, 1, 64), (2, 64, 64, 2, 2, 128),
    (1, 65, 65, 4, 2, 80), (1, 127, 129, 2, 1, 96), (2, 128, 128, 2, 2, 64), (1, 200, 257, 6, 2, 64), (1, 130, 130, 5, 1, 120),
    (1, 1, 1000, 8, 2, 128), (3, 1, 777, 12, 12, 64), (2, 4, 515, 8, 1, 64), (1, 5, 300, 16, 2, 128), (1, 300, 300, 1, 1, 16),
]
FORMS = [
    {}, {"cap": 10.0}, {"causal": True}, {"documents": "packed"}, {"slopes": True}, {"causal": True, "prefix": True, "cap": 20.0},
    {"documents": "mixed", "cap": 5.0, "slopes": True}, {"documents": "mixed", "causal": True, "prefix": True, "slopes": True},
    {"documents": "front", "causal": True},
]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_attention_against_the_definition(shape, form, dtype):
    import torch
    _case(torch, getattr(torch, dtype), *shape, seed=form, **FORMS[form])


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("shape", [(3, 40, 100, 6, 2, 48), (2, 64, 64, 4, 2, 64), (1, 32, 128, 4, 1, 40), (2, 1, 128, 128, 2, 64), (5, 128, 128, 3, 3, 64),
                                   (2, 97, 127, 2, 2, 56)], ids=lambda s: "x".join(map(str, s)))
def test_short_sequences(shape, form):
    import torch
    _case(torch, torch.bfloat16, *shape, **FORMS[form], seed=3)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("shape", [(3, 40, 60, 3, 3, 120), (2, 30, 50, 4, 2, 128), (2, 33, 64, 2, 2, 48), (2, 64, 64, 1, 1, 128), (2, 120, 128, 2, 2, 128),
                                   (2, 20, 100, 10, 2, 80)], ids=lambda s: "x".join(map(str, s)))
def test_short_sequences_of_each_width(shape, form, dtype):
    import torch
    _case(torch, getattr(torch, dtype), *shape, **FORMS[form], seed=4)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("w", [32, 128])
def test_one_key_has_no_score_gradient(w, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v, go = (torch.randn((3, 1, heads, w), generator=g, device="cuda").to(getattr(torch, dtype)) for heads in (4, 2, 2, 4))
    for form in (binding.attention_form(), binding.attention_form(cap=20.0, causal=True)):
        f = binding.mslt_attention(q, k, v, form)
        d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form)
        assert (d["dq"] == 0).all() and (d["dk"] == 0).all()
        # (out is p v / p, p being 2 to what rounding the maximum took off: off v by the roundings of the product and the quotient)
        want, _ = R.attention(q, k, v, cap=form.cap, causal=bool(form.causal), grad=go)
        for name in ("out", "dv"):
            R.check({**f, **d}[name], want[name], dtype == "bfloat16", name)


@pytest.mark.parametrize("shape", [(2, 2, 2, 2, 2, 64), (3, 4, 4, 4, 2, 128), (2, 7, 9, 2, 2, 32), (2, 32, 32, 4, 1, 64), (1, 31, 31, 2, 2, 120)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("form", [{}, {"causal": True, "cap": 10.0}, {"slopes": 0.1}])
def test_few_keys_round_gradients_once(shape, form):
    # Up to 32 keys the terms of a gradient go into its products in two bf16 parts.  What is left of a term is 2^-8 of what one part would
    # lose, and so is what the stored output's rounding leaves in delta (taken out with p in one part): the bounds of those
    # roundings times 2^-8, doubled for products of roundings, next to the gradient's own half step.
    import torch
    B, n, S, h, kv, w = shape
    g = torch.Generator(device="cuda").manual_seed(6)
    q, k, v, go = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((B, n, h, w), (B, S, kv, w), (B, S, kv, w), (B, n, h, w)))
    slopes = torch.full((h,), form["slopes"], device="cuda") if "slopes" in form else None
    f = {name: x for name, x in form.items() if name != "slopes"}
    a = binding.mslt_attention(q, k, v, binding.attention_form(**f), slopes=slopes)
    d = binding.mslt_attention_backward(q, k, v, a["out"], a["lse"], go, binding.attention_form(**f), slopes=slopes)
    want, _ = R.attention(q, k, v, grad=go, slopes=slopes, **f)
    for name in ("dq", "dk", "dv"):
        value, f32, b16 = want[name]
        own = 2.0 ** -8 * value.abs()
        R.check(d[name], (value, f32, (b16 - own) * 2.0 ** -7 + own), True, name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("form", [0, 5, 6])
@pytest.mark.parametrize("shape", [(32, 128, 128, 8, 8, 64), (40, 200, 200, 8, 8, 64), (64, 256, 256, 4, 4, 128), (70, 330, 350, 8, 4, 96),
                                   (64, 130, 130, 6, 6, 128)], ids=lambda s: "x".join(map(str, s)))
def test_batches_that_fill_the_chip(shape, form, dtype):
    """128 rows a workgroup and more: small batches are dealt out 32 rows at a time."""
    import torch
    _case(torch, getattr(torch, dtype), *shape, seed=form, **FORMS[form])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(1, 33, 16500, 1, 1, 8), (1, 2100, 2100, 8, 1, 16), (256, 1, 32900, 1, 1, 8), (1, 700, 2200, 2, 1, 64)],
                         ids=lambda s: "x".join(map(str, s)))
def test_more_tiles_than_one_list_holds(shape, dtype):
    import torch
    _case(torch, getattr(torch, dtype), *shape, documents="packed" if shape[2] < 4000 else None, causal=True, backward=shape[0] == 1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 150, 150, 4, 2, 64), (2, 20, 150, 2, 1, 128), (2, 1, 300, 4, 1, 64)], ids=lambda s: "x".join(map(str, s)))
def test_padding_may_hold_anything(shape, dtype):
    import torch
    for kind in ("packed", "mixed", "front"):
        got = _case(torch, getattr(torch, dtype), *shape, documents=kind, nan_padding=True, cap=8.0, slopes=True)
        dead = _documents(torch, shape[0], shape[2], kind, 0) < 0
        for name in ("dk", "dv"):
            assert (got[name][dead] == 0).all()
        for name in ("out", "dq"):
            assert (got[name][dead[:, shape[2] - shape[1]:]] == 0).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_large_scores_stay_finite(dtype):
    import torch
    # scores of some thousands without a cap: one key takes a row; with a cap the tanh saturates at both ends
    for cap in (0.0, 30.0):
        dt = getattr(torch, dtype)
        g = torch.Generator(device="cuda").manual_seed(1)
        q, k, v, go = (torch.randn((1, 70, 2, 64), generator=g, device="cuda").mul(s).to(dt) for s in (60, 60, 1, 1))
        form = binding.attention_form(cap=cap)
        f = binding.mslt_attention(q, k, v, form)
        d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form)
        want, _ = R.attention(q, k, v, cap=cap, grad=go)
        for name, w3 in want.items():
            R.check({**f, **d}[name], w3, dt == torch.bfloat16, name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 70, 70, 4, 2, 64), (1, 1, 2000, 4, 2, 128), (64, 128, 128, 8, 8, 64), (64, 260, 260, 4, 4, 128)],
                         ids=lambda s: "x".join(map(str, s)))
def test_what_is_not_a_number_stays_so(shape, dtype):
    import torch
    B, n, S, h, kv, w = shape
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(s, generator=g, device="cuda").to(dt) for s in ((B, n, h, w), (B, S, kv, w), (B, S, kv, w)))
    q[0, n // 2, 1, 3] = float("nan")
    for cap in (0.0, 30.0):
        form = binding.attention_form(cap=cap)
        f = binding.mslt_attention(q, k, v, form)
        d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], torch.ones_like(q), form)
        bad = torch.zeros((B, n, h), dtype=torch.bool, device="cuda")
        bad[0, n // 2, 1] = True
        assert torch.equal(bad, torch.isnan(f["lse"]).transpose(1, 2))
        for x in (f["out"], d["dq"]):
            assert torch.equal(bad[..., None].expand_as(x), torch.isnan(x))
        for x in (d["dk"], d["dv"]):      # its kv head's
            assert torch.isnan(x[0, :, 1 // (h // kv)]).all() and not torch.isnan(x[1:]).any()


def test_a_cap_far_above_the_scores():
    # Scores of some tens under a cap of 10^5: what the cap takes off is below 10^-5 of them, and no more may get lost than without a
    # cap.  The bounds are those without (16 roundings of a score's terms): the polynomial adds five and what it leaves out, one.
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v, go = (torch.randn((2, 90, 2, 64), generator=g, device="cuda").mul(s) for s in (3, 3, 1, 1))
    form = binding.attention_form(cap=1e5, scale=0.25)
    f = binding.mslt_attention(q, k, v, form)
    d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form)
    want, _ = R.attention(q, k, v, cap=1e5, scale=0.25, grad=go)
    bounds, _ = R.attention(q, k, v, scale=0.25, grad=go)
    for name in want:
        R.check({**f, **d}[name], (want[name][0], *bounds[name][1:]), False, name)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_layouts(dtype):
    """Heads before tokens, rows apart, a batch that is broadcast, results into parts of a packed tensor: the same values."""
    import torch
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    B, S, h, kv, w = 2, 90, 4, 2, 64
    q, k, v, go = (torch.randn(s, generator=g, device="cuda").to(dt) for s in ((B, S, h, w), (1, S, kv, w), (B, S, kv, w), (B, S, h, w)))
    k = k.expand(B, S, kv, w)
    form = binding.attention_form(cap=15.0, causal=True)
    f = binding.mslt_attention(q, k.contiguous(), v, form)
    d = binding.mslt_attention_backward(q, k.contiguous(), v, f["out"], f["lse"], go, form)
    head_major = lambda x: x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    apart = torch.zeros(B, S + 3, h, w + 16, dtype=dt, device="cuda")
    apart[:, :S, :, :w] = go
    packed = torch.full((B, S + 1, (h + 2 * kv) * w), 7.0, dtype=dt, device="cuda")
    part = lambda at, heads: packed[:, :S, at * w:(at + heads) * w].view(B, S, heads, w)
    out2 = torch.full((B, h, S + 1, w), 7.0, dtype=dt, device="cuda")
    f2 = binding.mslt_attention(head_major(q), k, head_major(v), form, out=out2[:, :, :S].permute(0, 2, 1, 3))
    d2 = binding.mslt_attention_backward(head_major(q), k, head_major(v), f2["out"], f2["lse"], apart[:, :S, :, :w], form,
                                         grads=(part(0, h), part(h, kv), part(h + kv, kv)))
    for name, want in {**f, **d}.items():
        assert torch.equal({**f2, **d2}[name], want), name
    assert (packed[:, S:] == 7).all() and (out2[:, :, S:] == 7).all()        # rows behind the last one stay as they were


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 140, 140, 4, 2, 64), (2, 3, 140, 4, 2, 128), (2, 90, 90, 4, 2, 64)], ids=lambda s: "x".join(map(str, s)))
def test_offsets_beyond_32_bits(shape, dtype):
    """Rows as far apart as they may be, heads and sequences 2^31 and 2^32 elements apart."""
    import torch
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(7)
    B, n, S, h, kv, w = shape
    far = (1 << 32, 1 << 22, 1 << 31)
    room = torch.empty((1 << 32) + (1 << 31) + S * (1 << 22), dtype=dt, device="cuda")

    def spread(x, at, strides):
        y = room.as_strided(x.shape, (*strides, 1), at)
        y.copy_(x)
        return y

    q, k, v, go = (torch.randn(s, generator=g, device="cuda").to(dt) for s in ((B, n, h, w), (B, S, kv, w), (B, S, kv, w), (B, n, h, w)))
    form = binding.attention_form(cap=15.0, causal=True)
    f = binding.mslt_attention(q, k, v, form)
    d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form)
    near = (1 << 32, 1 << 22, 1 << 12)
    q2, go2 = spread(q, 1024, near), spread(go, 1 << 20, near)
    k2, v2 = spread(k, 0, far), spread(v, 256, far)
    grads = tuple(room.as_strided(x.shape, (*far, 1), at) for x, at in ((k, 512), (v, 768)))
    f2 = binding.mslt_attention(q2, k2, v2, form)
    d2 = binding.mslt_attention_backward(q2, k2, v2, f2["out"], f2["lse"], go2, form, grads=(torch.empty_like(q), *grads))
    for name, want in {**f, **d}.items():
        assert torch.equal({**f2, **d2}[name], want), name


@pytest.mark.parametrize("n", [1, 90])
def test_same_values_every_time_on_any_stream_and_in_graphs(n):
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    B, S, h, kv, w = 2, 1500, 4, 2, 64
    q, go = (torch.randn((B, n, h, w), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((B, S, kv, w), generator=g, device="cuda").bfloat16() for _ in range(2))
    docs = _documents(torch, B, S, "front", 0)
    form = binding.attention_form(cap=30.0, causal=True)

    def step(**kw):
        f = binding.mslt_attention(q, k, v, form, documents=docs, **kw)
        return {**f, **binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form, documents=docs, **kw)}

    want = {name: t.clone() for name, t in step().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for name in want:
        assert torch.equal(got[name], want[name]), name
    graphs = []
    for _ in range(2):          # two graphs of the same operands, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = step()
        graphs.append((graph, res))
    for i in range(6):
        graph, res = graphs[i % 2]
        for t in res.values():
            t.fill_(3.0)
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(res[name], want[name]) and torch.equal(eager[name], want[name]), name


def test_gradients_against_differences():
    """fp32, a cap, a bias and masks together: the gradients against central differences of the output in float64."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    q, k, v, go = (torch.randn(s, generator=g, device="cuda") for s in ((1, 9, 2, 8), (1, 12, 1, 8), (1, 12, 1, 8), (1, 9, 2, 8)))
    masks = {"documents": torch.tensor([[0, 0, 0, 0, 0, 1, 1, 1, 1, 1, 1, -1]], dtype=torch.int32, device="cuda"),
             "prefix": torch.tensor([7], dtype=torch.int32, device="cuda"), "slopes": torch.tensor([0.1, -0.05], device="cuda")}
    kw = {"cap": 3.0, "causal": True}
    form = binding.attention_form(**kw)
    f = binding.mslt_attention(q, k, v, form, **masks)
    d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form, **masks)
    loss = lambda *x: (R.attention(*x, **kw, **masks)[0]["out"][0] * go.double()).sum()
    x = [t.double() for t in (q, k, v)]
    step = 2.0 ** -13        # differences are off by its square, 2^-26, times third derivatives of order ten
    for i, name in enumerate(("dq", "dk", "dv")):
        for e in range(0, x[i].numel(), 5):
            hi, lo = [t.clone() for t in x], [t.clone() for t in x]
            hi[i].view(-1)[e] += step
            lo[i].view(-1)[e] -= step
            slope = ((loss(*hi) - loss(*lo)) / (2 * step)).item()
            assert abs(d[name].reshape(-1)[e].item() - slope) < 2.0 ** -16, (name, e)


@pytest.mark.parametrize("shape", [(64, 32, 32, 32, 4, 64), (64, 32, 32, 64, 8, 64), (24, 32, 32, 32, 4, 128), (64, 32, 32, 32, 4, 128), (130, 9, 30, 64, 4, 80),
                                   (2, 32, 32, 64, 1, 64)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("form", [{}, {"causal": True, "cap": 10.0}, {"slopes": 0.1}])
def test_few_keys_round_gradients_once_in_any_batch(shape, form):
    # More than 128 rows to a kv head, from batches that leave compute units idle to ones that fill the chip: the bounds of
    # test_few_keys_round_gradients_once, which hold whatever the batch.
    import torch
    B, n, S, h, kv, w = shape
    g = torch.Generator(device="cuda").manual_seed(6)
    q, k, v, go = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((B, n, h, w), (B, S, kv, w), (B, S, kv, w), (B, n, h, w)))
    slopes = torch.full((h,), form["slopes"], device="cuda") if "slopes" in form else None
    f = {name: x for name, x in form.items() if name != "slopes"}
    a = binding.mslt_attention(q, k, v, binding.attention_form(**f), slopes=slopes)
    d = binding.mslt_attention_backward(q, k, v, a["out"], a["lse"], go, binding.attention_form(**f), slopes=slopes)
    want, _ = R.attention(q, k, v, grad=go, slopes=slopes, **f)
    for name in ("dq", "dk", "dv"):
        value, f32, b16 = want[name]
        own = 2.0 ** -8 * value.abs()
        R.check(d[name], (value, f32, (b16 - own) * 2.0 ** -7 + own), True, name)


def test_as_part_of_a_torch_graph():
    """Wrapped into an autograd.Function, whose forward and backward run with gradients off; leaves are refused outside of one."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(12)
    leaves = [torch.randn(s, generator=g, device="cuda", requires_grad=True) for s in ((2, 50, 4, 32), (2, 50, 2, 32), (2, 50, 2, 32))]
    form = binding.attention_form(causal=True)

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            f = binding.mslt_attention(q, k, v, form)
            ctx.save_for_backward(q, k, v, f["out"], f["lse"])
            return f["out"]

        @staticmethod
        def backward(ctx, grad):
            d = binding.mslt_attention_backward(*ctx.saved_tensors, grad.contiguous(), form)
            return d["dq"], d["dk"], d["dv"]

    go = torch.randn(leaves[0].shape, generator=g, device="cuda")
    (Attention.apply(*leaves) * go).sum().backward()
    want, _ = R.attention(*(x.detach() for x in leaves), causal=True, grad=go)
    for x, name in zip(leaves, ("dq", "dk", "dv")):
        R.check(x.grad, want[name], False, name)
    with pytest.raises(binding.MsltError, match="requires a gradient"):
        binding.mslt_attention(*leaves, form)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 90, 90, 4, 2, 64), (3, 60, 60, 2, 2, 128), (1, 400, 400, 6, 2, 64), (40, 200, 200, 8, 8, 64), (2, 3, 300, 4, 2, 128)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_rows_that_see_one_key_among_many(shape, cap, dtype):
    # The gradient of a single score is zero.  Exactly so in the first row of a causal sequence.  Documents of one token leave roundings:
    # fp32's; in bf16 dP - delta is off by half a step of the stored output, 2^-8 of the size of dO O, of which the mended delta
    # takes off all but what rounding that to bf16 leaves, 2^-8 of it: 2^-16, where forms_reference's b16 counts 2^-7 for delta
    # (and twice the probability's).  Doubled for products of roundings: b16 times 2^-8.
    import torch
    dt = getattr(torch, dtype)
    B, n, S, h, kv, w = shape
    g = torch.Generator(device="cuda").manual_seed(13)
    q, k, v, go = (torch.randn(s, generator=g, device="cuda").mul(1.5).to(dt) for s in ((B, n, h, w), (B, S, kv, w), (B, S, kv, w), (B, n, h, w)))
    form = binding.attention_form(cap=cap, causal=True)
    if n == S:
        f = binding.mslt_attention(q, k, v, form)
        d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form)
        assert (d["dq"][:, 0] == 0).all()
        want, _ = R.attention(q, k, v, cap=cap, causal=True, grad=go)
        for name in ("dq", "dk", "dv"):
            R.check(d[name], want[name], dt == torch.bfloat16, name)
    docs = torch.arange(S, dtype=torch.int32, device="cuda").expand(B, S).contiguous()
    form = binding.attention_form(cap=cap)
    f = binding.mslt_attention(q, k, v, form, documents=docs)
    d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form, documents=docs)
    want, _ = R.attention(q, k, v, cap=cap, documents=docs, grad=go)
    for name in ("dq", "dk"):
        value, f32, b16 = want[name]
        assert (value.abs() <= f32).all()      # (zero but for float64's own roundings)
        R.check(d[name], (value, f32, b16 * 2.0 ** -8), dt == torch.bfloat16, name)


@pytest.mark.parametrize("dtype,cap", [("float32", 400.0), ("float32", 3000.0), ("bfloat16", 30000.0)])
@pytest.mark.parametrize("shape", [(2, 90, 90, 2, 2, 64), (1, 64, 64, 2, 2, 128), (1, 300, 300, 4, 2, 64), (1, 3, 700, 4, 2, 64)], ids=lambda s: "x".join(map(str, s)))
def test_scores_near_the_cap_leave_others_their_digits(shape, cap, dtype):
    # Every seventh query's scores reach the cap, all others are some tens at most: those may be off by what they are off without a cap
    # (16 roundings of a score's terms, to which the polynomial adds six) and in bf16 by its own roundings; not by roundings of the cap.
    import torch
    dt = getattr(torch, dtype)
    B, n, S, h, kv, w = shape
    g = torch.Generator(device="cuda").manual_seed(14)
    q, k, v, go = (torch.randn(s, generator=g, device="cuda").mul(1.5) for s in ((B, n, h, w), (B, S, kv, w), (B, S, kv, w), (B, n, h, w)))
    large = torch.arange(n, device="cuda") % 7 == 1
    q[:, large] *= cap / 3
    go[:, large] = 0
    q, k, v, go = (x.to(dt) for x in (q, k, v, go))
    form = binding.attention_form(cap=cap)
    f = binding.mslt_attention(q, k, v, form)
    d = binding.mslt_attention_backward(q, k, v, f["out"], f["lse"], go, form)
    want, lse = R.attention(q, k, v, cap=cap, grad=go)
    plain = q.clone()
    plain[:, large] = 0
    bounds, _ = R.attention(plain, k, v, grad=go)
    for name in ("out", "dq"):
        R.check({**f, **d}[name][:, ~large], tuple(x[:, ~large] for x in (want[name][0], *bounds[name][1:])), dt == torch.bfloat16, name)
    # the log-sum-exp: of scores whose terms add up to less than 2^7, 32 roundings of that
    assert ((f["lse"].double() - lse)[:, :, ~large].abs() <= 32 * 2.0 ** -24 * 2 ** 7).all()
