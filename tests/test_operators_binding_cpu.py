"""What the binding of the operators between the QKV projection and the output projection refuses before it looks at a device."""
import pytest

from paper_2011_13635_amd import binding as b

ROT, ATT = b.rotary_form(64), b.attention_form()


def _calls(torch, **changes):
    """(name, call) of every operator on tensors of one shape, with some operands replaced."""
    x = {n: torch.zeros(1, 2, 2, 64) for n in ("q", "k", "v", "grad_q", "grad_k", "out", "grad_out")}
    x.update(gain_q=torch.ones(64), gain_k=torch.ones(64), lse=torch.zeros(1, 2, 2), rot=ROT, att=ATT, slopes=None)
    x.update(changes)
    norm = (x["q"], x["k"], x["gain_q"], x["gain_k"], 1e-6, x["rot"])
    return {
        "mslt_rotary": lambda: b.mslt_rotary(x["q"], x["k"], x["rot"]),
        "mslt_head_norm_rotary": lambda: b.mslt_head_norm_rotary(*norm),
        "mslt_head_norm_rotary_backward": lambda: b.mslt_head_norm_rotary_backward(*norm, x["grad_q"], x["grad_k"]),
        "mslt_attention": lambda: b.mslt_attention(x["q"], x["k"], x["v"], x["att"], slopes=x["slopes"]),
        "mslt_attention_backward": lambda: b.mslt_attention_backward(x["q"], x["k"], x["v"], x["out"], x["lse"], x["grad_out"], x["att"],
                                                                     slopes=x["slopes"]),
    }


NEEDS = {
    "mslt_rotary": ("q", "rot"),      # (k may be left out)
    "mslt_head_norm_rotary": ("q", "k", "gain_q", "gain_k", "rot"),
    "mslt_head_norm_rotary_backward": ("q", "k", "gain_q", "gain_k", "grad_q", "grad_k", "rot"),
    "mslt_attention": ("q", "k", "v", "att"),
    "mslt_attention_backward": ("q", "k", "v", "out", "lse", "grad_out", "att"),
}


@pytest.mark.parametrize("name,operand", [(n, o) for n, needs in NEEDS.items() for o in needs])
def test_an_operand_that_is_missing(name, operand):
    import torch
    what = "form" if operand in ("rot", "att") else operand
    with pytest.raises(b.MsltError, match=f"{name}: {what} must be"):
        _calls(torch, **{operand: None})[name]()


OPERANDS = {**NEEDS, "mslt_rotary": ("q", "k", "rot"), "mslt_attention": ("q", "k", "v", "slopes"),
            "mslt_attention_backward": (*NEEDS["mslt_attention_backward"], "slopes")}


@pytest.mark.parametrize("name,operand", [(n, o) for n, needs in OPERANDS.items() for o in needs if o not in ("rot", "att")])
def test_a_gradient_that_would_be_lost(name, operand):
    import torch
    shape = {"gain_q": (64,), "gain_k": (64,), "lse": (1, 2, 2), "slopes": (2,)}.get(operand, (1, 2, 2, 64))
    call = _calls(torch, **{operand: torch.ones(shape, requires_grad=True)})[name]
    with pytest.raises(b.MsltError, match=f"{name}: {operand} requires a gradient"):
        call()
    with torch.no_grad(), pytest.raises(b.MsltError, match="on a GPU"):      # (no further than the device, here)
        call()
