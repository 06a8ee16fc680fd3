"""Refusals of the operators between the QKV projection and the output projection: every check of the C entries on the host,
before anything is enqueued (no GPU is needed: addresses are made up and never read), and the binding's own."""
import ctypes as C

import pytest

from paper_2011_13635_amd import binding as b

AT = 0x10000


def _heads(rows=4, heads=2, width=64, at=AT, **changes):
    h = b.Heads(at, rows * heads * width, heads * width, width)
    for name, value in changes.items():
        setattr(h, name, value)
    return h


def _refused(rc, text):
    assert rc == b.MSLT_ERR_ARG
    message = b.load_library().mslt_last_error().decode()
    assert text in message, message


ATT = {"precision": 1, "batch": 2, "queries": 4, "keys": 4, "heads": 2, "kv_heads": 2, "width": 64}


def _attention(sizes=None, form=None, backward=False, workspace=AT, room=1 << 30, lse=AT, **operands):
    s = {**ATT, **(sizes or {})}
    lib = b.load_library()
    f = b.AttentionForm(0.125, 0.0, 0, None, None, None)
    for name, value in (form or {}).items():
        setattr(f, name, value)
    x = {n: C.byref(_heads()) for n in ("q", "k", "v", "out", "grad_out", "dq", "dk", "dv")}
    x.update({n: None if v is None else C.byref(v) for n, v in operands.items()})
    head = (None, *s.values(), x["q"], x["k"], x["v"])
    if backward:
        return lib.mslt_attention_backward(*head, x["out"], lse, x["grad_out"], C.byref(f), x["dq"], x["dk"], x["dv"], workspace, room)
    return lib.mslt_attention(*head, C.byref(f), x["out"], lse, workspace, room)


@pytest.mark.parametrize("sizes,text", [
    ({"precision": 2}, "precision"), ({"batch": 0}, "queries"), ({"queries": 0}, "queries"), ({"queries": 5}, "queries <= keys"),
    ({"kv_heads": 0}, "kv_heads"), ({"heads": 3}, "multiple of kv_heads"), ({"width": 0}, "needs"), ({"width": 136}, "at most 128"),
    ({"width": 60}, "16 bytes"), ({"precision": 0, "width": 62}, "16 bytes"), ({"keys": (1 << 24) + 1}, "2^24"),
    ({"batch": 1 << 20, "heads": 4, "kv_heads": 4}, "2^20")])
@pytest.mark.parametrize("backward", [False, True])
def test_attention_sizes(sizes, text, backward):
    _refused(_attention(sizes, backward=backward), text)
    n = C.c_size_t()
    _refused(b.load_library().mslt_attention_workspace(*{**ATT, **sizes}.values(), int(backward), C.byref(n)), text)


@pytest.mark.parametrize("form,text", [({"scale": 0.0}, "scale"), ({"scale": float("nan")}, "scale"), ({"scale": float("inf")}, "scale"),
                                       ({"cap": -1.0}, "cap"), ({"cap": float("nan")}, "cap"), ({"prefix": AT}, "causal")])
@pytest.mark.parametrize("backward", [False, True])
def test_attention_forms(form, text, backward):
    _refused(_attention(form=form, backward=backward), text)


@pytest.mark.parametrize("operand,backward", [("q", 0), ("k", 0), ("v", 0), ("out", 0), ("q", 1), ("k", 1), ("v", 1), ("out", 1), ("grad_out", 1),
                                              ("dq", 1), ("dk", 1), ("dv", 1)])
def test_attention_operands(operand, backward):
    _refused(_attention(backward=backward, **{operand: None}), "is null")
    _refused(_attention(backward=backward, **{operand: _heads(at=0)}), "is null")
    _refused(_attention(backward=backward, **{operand: _heads(at=AT + 8)}), "aligned")
    _refused(_attention(backward=backward, **{operand: _heads(row_stride=132)}), "multiple of 16 bytes")
    _refused(_attention(backward=backward, **{operand: _heads(batch_stride=-512)}), "outside")
    if operand in ("dq", "dk", "dv") or (operand == "out" and not backward):
        _refused(_attention(backward=backward, **{operand: _heads(batch_stride=0)}), "overlaps")
        _refused(_attention(backward=backward, **{operand: _heads(head_stride=56)}), "overlaps")
    _refused(_attention(backward=backward, lse=None), "lse")
    _refused(_attention(backward=backward, workspace=None), "workspace")
    _refused(_attention(backward=backward, workspace=AT + 4), "workspace")
    _refused(_attention(backward=backward, room=8), "workspace")


@pytest.mark.parametrize("sizes,text", [
    ({"heads": 65, "kv_heads": 1}, "64 heads"), ({"batch": 1 << 18, "queries": 1 << 12, "keys": 1 << 12, "kv_heads": 1}, "2^30 queries"),
    ({"batch": 1 << 15, "queries": 1, "keys": 1 << 14}, "2^29 keys")])
@pytest.mark.parametrize("backward", [False, True])
def test_attention_limits(sizes, text, backward):
    s = {**ATT, **sizes}
    _refused(_attention(sizes, backward=backward), text)
    n = C.c_size_t()
    _refused(b.load_library().mslt_attention_workspace(*s.values(), int(backward), C.byref(n)), text)
    # one step inside them
    inside = {"heads": 64} if s["heads"] == 65 else {"batch": s["batch"] // 2}
    assert b.load_library().mslt_attention_workspace(*{**s, **inside}.values(), int(backward), C.byref(n)) == 0


@pytest.mark.parametrize("form", [{"scale": 2.0 ** -21}, {"scale": 2.0 ** 21}, {"scale": 1.0, "cap": 2.0 ** -17}, {"scale": 1.0, "cap": 2.0 ** 25}])
def test_attention_factors_out_of_range(form):
    _refused(_attention(form=form), "2^")
    _refused(_attention(form=form, backward=True), "2^")


def test_attention_strides_out_of_reach():
    far = (1 << 22) + 8
    for name in ("k", "v"):
        for backward in (False, True):
            _refused(_attention(backward=backward, **{name: _heads(row_stride=far)}), "2^22")
    grouped = {"heads": 4, "kv_heads": 2}
    for name in ("q", "grad_out"):
        _refused(_attention(backward=True, **{name: _heads(row_stride=far)}), "2^22")
        _refused(_attention(grouped, backward=True, **{name: _heads(head_stride=(1 << 27) + 8)}), "2^28")


def test_attention_workspace_counts_split_keys_and_rows():
    n, f, g = C.c_size_t(), C.c_size_t(), C.c_size_t()
    lib = b.load_library()
    assert lib.mslt_attention_workspace(1, 1, 1, 65536, 8, 1, 64, 0, C.byref(n)) == 0
    assert lib.mslt_attention_workspace(1, 64, 128, 128, 16, 16, 64, 0, C.byref(f)) == 0
    assert lib.mslt_attention_workspace(1, 64, 128, 128, 16, 16, 64, 1, C.byref(g)) == 0
    assert n.value > 8 * 64 * 4 * 2 and f.value < 1 << 16 and g.value >= 64 * 16 * 128 * 4
    _refused(lib.mslt_attention_workspace(1, 1, 1, 1, 1, 1, 64, 0, None), "null")


ROT = {"precision": 0, "batch": 2, "seq": 4, "q_heads": 2, "k_heads": 2, "width": 64}


def _rotary(which, sizes=None, form=None, gain=AT, eps=1e-6, workspace=AT, room=1 << 30, dgain=AT, **operands):
    s = {**ROT, **(sizes or {})}
    lib = b.load_library()
    f = b.rotary_form(64)
    for name, value in (form or {}).items():
        setattr(f, name, value)
    x = {n: C.byref(_heads()) for n in ("q", "k", "q_out", "k_out", "grad_q", "grad_k", "dq", "dk")}
    x.update({n: None if v is None else C.byref(v) for n, v in operands.items()})
    head = (None, *s.values(), x["q"], x["k"])
    if which == "rotary":
        return lib.mslt_rotary(*head, None, C.byref(f), 0, x["q_out"], x["k_out"])
    head = (*head, gain, AT, 0, eps, None, C.byref(f))
    if which == "norm":
        return lib.mslt_head_norm_rotary(*head, x["q_out"], x["k_out"])
    return lib.mslt_head_norm_rotary_backward(*head, x["grad_q"], x["grad_k"], x["dq"], x["dk"], dgain, AT, workspace, room)


WHICH = ("rotary", "norm", "backward")


@pytest.mark.parametrize("which", WHICH)
def test_rotary_refusals(which):
    for sizes in ({"precision": 3}, {"batch": 0}, {"seq": 0}, {"q_heads": 0}, {"width": 0}, {"width": 257}, {"k_heads": -1}, {"batch": 1 << 16, "seq": 1 << 16}):
        _refused(_rotary(which, sizes), "")
    _refused(_rotary(which, {"k_heads": 0}), "k without heads")
    nan, inf = float("nan"), float("inf")
    for form, text in (({"rotary_width": 63}, "rotary_width"), ({"rotary_width": 66}, "rotary_width"), ({"rotary_width": -2}, "rotary_width"),
                       ({"scaling": 3}, "scaling"), ({"theta": 1.0}, "theta"), ({"theta": nan}, "theta"), ({"magnitude": inf}, "magnitude"),
                       ({"scaling": 1, "factor": 0.0}, "factor"), ({"scaling": 2, "factor": 2.0, "original_length": 0.0}, "original_length"),
                       ({"scaling": 2, "factor": 2.0, "original_length": 64.0, "low_turns": 4.0, "high_turns": 4.0}, "low_turns")):
        _refused(_rotary(which, form=form), text)
    inputs, outputs = {"rotary": (("q", "k"), ("q_out", "k_out")), "norm": (("q", "k"), ("q_out", "k_out")),
                       "backward": (("q", "k", "grad_q", "grad_k"), ("dq", "dk"))}[which]
    for name in inputs + outputs:
        if (which, name) != ("rotary", "k"):
            _refused(_rotary(which, **{name: None}), "")
        _refused(_rotary(which, **{name: _heads(at=0)}), "is null")
        _refused(_rotary(which, **{name: _heads(at=AT + 2)}), "aligned")
        _refused(_rotary(which, **{name: _heads(row_stride=-1)}), "outside")
    for name in outputs:
        _refused(_rotary(which, **{name: _heads(batch_stride=0)}), "overlaps")
        _refused(_rotary(which, **{name: _heads(head_stride=32)}), "overlaps")


def test_norm_refusals():
    for which in ("norm", "backward"):
        _refused(_rotary(which, gain=None), "gain")
        for eps in (-1.0, float("nan"), float("inf")):
            _refused(_rotary(which, eps=eps), "eps")
    _refused(_rotary("backward", dgain=None), "gain")
    _refused(_rotary("backward", workspace=None), "workspace")
    _refused(_rotary("backward", room=16), "workspace")
    n = C.c_size_t()
    lib = b.load_library()
    _refused(lib.mslt_head_norm_workspace(1, 1, 1, 1, 64, None), "null")
    assert lib.mslt_head_norm_workspace(1, 1, 1, 1, 64, C.byref(n)) == 0 and n.value >= 2 * 64 * 4


def test_binding_refuses():
    import torch
    x = torch.zeros(1, 2, 2, 64)
    with pytest.raises(b.MsltError, match="on a GPU"):
        b.mslt_rotary(x, x, b.rotary_form(64))
    with pytest.raises(b.MsltError, match="on a GPU"):
        b.mslt_attention(x, x, x, b.attention_form())
    with pytest.raises(b.MsltError, match="scaling"):
        b.rotary_form(64, scaling="other")
    with pytest.raises(b.MsltError, match="scale"):
        b.attention_form(scale=0.0)
    with pytest.raises(b.MsltError, match="fp32 tensors"):
        b._precision("f", x.half())
    for t, kw in ((x[0], {}), (x, {"like": x.double()}), (x, {"shape": torch.Size((1, 2, 2, 32))}), (x.transpose(2, 3), {})):
        with pytest.raises(b.MsltError):
            b._heads("f", "x", t, **kw)
    for t in (torch.zeros(4), torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(b.MsltError):
            b._flat("f", "x", t, torch.int32, (4,))
    form, none = b.attention_form(), x[..., :0]
    assert b._attention_call("f", none, none, none, form, None, None, None)[0][-1] == 0        # (the library refuses the width)
    with pytest.raises(b.MsltError):
        b._rotary_sizes("f", x, torch.zeros(1, 3, 2, 64))
