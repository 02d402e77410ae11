"""Gated feed-forward block with infinite operands, at even and odd widths: infinities where the formulas have them, not NaN.  Operands are positive, so that no
sum of the formulas meets infinities of both signs, and the row that is infinite is the only one."""
import pytest
import torch


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


def positive(rows, d, f, bf16):
    g = torch.Generator().manual_seed(rows + d)
    rnd = lambda *s: 0.5 + torch.rand(*s, generator=g)  # noqa: E731
    dt = torch.bfloat16 if bf16 else torch.float32
    return [t.to(dt).cuda() for t in (rnd(rows, d), rnd(2 * f, d) / d, rnd(d, f) / f, rnd(rows, d))]


SIZES = [(3, 64, 128), (3, 33, 17), (70, 40, 31), (70, 31, 40), (700, 129, 65), (700, 128, 67)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d,f", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", ["SB_ACT_RELU", "SB_ACT_SILU", "SB_ACT_GELU"])
def test_forward(rows, d, f, bf16, act):
    b = sb()
    x, wgu, wd, _ = positive(rows, d, f, bf16)
    y = b.ffn_forward(x, wgu, wd, getattr(b, act))
    x[1, 2] = float("inf")
    z, gu = b.ffn_forward(x, wgu, wd, getattr(b, act), save=True)
    b.ops_check()
    rest = [i for i in range(rows) if i != 1]
    assert torch.isfinite(y).all() and torch.equal(z[rest], y[rest])
    assert (gu[1] == float("inf")).all() and (z[1] == float("inf")).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d,f", SIZES)
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", ["SB_ACT_RELU", "SB_ACT_SILU", "SB_ACT_GELU"])
def test_backward(rows, d, f, bf16, act):
    """dy infinite in one place: dH's row, and with it dG, dU and dx's row, are infinite (a' is positive); every entry of dWgu takes up an infinite product;
    of dWd the row of that column."""
    b = sb()
    kind = getattr(b, act)
    x, wgu, wd, dy = positive(rows, d, f, bf16)
    _, gu = b.ffn_forward(x, wgu, wd, kind, save=True)
    one = b.ffn_backward(dy, x, gu, wgu, wd, kind)
    dy[1, 2] = float("inf")
    dx, dwgu, dwd = b.ffn_backward(dy, x, gu, wgu, wd, kind)
    b.ops_check()
    rest = [i for i in range(rows) if i != 1]
    assert all(torch.isfinite(t).all() for t in one) and torch.equal(dx[rest], one[0][rest])
    assert (dx[1] == float("inf")).all() and (dwgu == float("inf")).all()
    cols = [i for i in range(d) if i != 2]
    assert (dwd[2] == float("inf")).all() and torch.equal(dwd[cols], one[2][cols])
