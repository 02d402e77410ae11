"""Gated feed-forward block in bf16 where the activation is small: H and its gradients keep their relative precision along the negative tail.  A second product
by the identity (and a gradient of units) hands H, dG and dU out one by one."""
import pytest
import torch


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


F = 128


def gates(rows):
    """[rows, F] gates between -9 and 3, exact in bf16, and the operands that make them: x = [gates, ones], a gate's weights pick its column, up's the ones"""
    g = torch.linspace(-9, 3, rows * F, dtype=torch.float64).view(F, rows).t().contiguous().bfloat16()
    x = torch.cat([g, torch.ones(rows, F, dtype=torch.bfloat16)], 1).cuda()
    eye, none = torch.eye(F), torch.zeros(F, F)
    wgu = torch.cat([torch.cat([eye, none], 1), torch.cat([none, eye], 1)], 0).bfloat16().cuda()
    wd = torch.cat([eye, none], 0).bfloat16().cuda()                    # y = [H, 0]
    return g.double().cuda(), x, wgu, wd


def formulas(g, kind, b):
    if kind == b.SB_ACT_SILU:
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    cdf = 0.5 * torch.erfc(-g / 2 ** 0.5)
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / (2 * torch.pi) ** 0.5


# H is rounded to bf16 as an operand (half a step, 2^-8 of the value) and out of a product by one exactly.  The activation's own error is that of its
# approximations: exp of an argument of up to 41 (g = -9), whose rounding is 41 * 2^-23, and its quotient, polynomial and products, a few times 2^-23: 2^-16 in all.
REL = 2.0 ** -8 + 2.0 ** -16


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [5, 60, 700])
@pytest.mark.parametrize("act", ["SB_ACT_GELU", "SB_ACT_SILU"])
def test_small_activations_keep_their_precision(rows, act):
    b = sb()
    kind = getattr(b, act)
    g, x, wgu, wd = gates(rows)
    y, gu = b.ffn_forward(x, wgu, wd, kind, save=True)
    assert torch.equal(gu[:, :F].double(), g)
    a, da = formulas(g, kind, b)
    assert ((y[:, :F].double() - a).abs() <= REL * a.abs()).all()
    # backward: dH is one everywhere; dX = [dG, dU], through the identity
    dy = torch.cat([torch.ones(rows, F), torch.zeros(rows, F)], 1).bfloat16().cuda()
    dx = b.ffn_backward(dy, x, gu, wgu, wd, kind, needs=(True, False, False))[0].double()
    assert ((dx[:, F:] - a).abs() <= REL * a.abs()).all()
    # a' is a sum whose parts cancel near its zero (-0.75 and -1.28): relative to the parts
    size = da.abs() + (a / g).abs() + (da - a / g).abs()
    assert ((dx[:, :F] - da).abs() <= 2.0 ** -8 * da.abs() + 2.0 ** -16 * size).all()
    b.ops_check()
