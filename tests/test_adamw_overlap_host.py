"""What a step of AdamW writes must not overlap: refused by the binding's first step (on the CPU, where a call that comes so far is refused for its device)."""
import pytest


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


def lists(torch):
    p = [torch.zeros(64), torch.zeros(32), torch.zeros(0)]
    return p, [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]


def step(b, message, *args, **kw):
    opt = b.AdamW(*args, **kw)
    with pytest.raises(b.SBError, match=message):
        opt.step(1e-3)


def test_overlapping_tensors_are_refused():
    import torch
    b = sb()
    p, g, m, v = lists(torch)
    step(b, "CUDA device", p, g, m, v)                                    # neighbours, and empty tensors, are fine
    room = torch.zeros(96)
    step(b, "CUDA device", [room[:64], room[64:], p[2]], g, m, v)
    step(b, "overlap", [room[:64], room[63:95], p[2]], g, m, v)
    step(b, "overlap", p, g, m, [m[0], v[1], v[2]])                        # one tensor for both moments
    step(b, "overlap", p, g, [m[0], m[0][:32], m[2]], v)                   # one moment for two parameters
    step(b, "overlap", p, g, [p[0], m[1], m[2]], v)
    step(b, "overlap", p, g, m, v, shadows=[m[1].view(torch.bfloat16), p[1].bfloat16(), p[2].bfloat16()])


def test_overlapping_scales_are_refused():
    import torch
    b = sb()
    p, g = [torch.zeros(300), torch.zeros(300)], [torch.zeros(300), torch.zeros(300)]
    m, v = ([torch.zeros(300, dtype=torch.uint8) for _ in p] for _ in range(2))
    s = torch.zeros(8)
    step(b, "CUDA device", p, g, m, v, [s[:2], s[2:4]], [s[4:6], s[6:]])
    step(b, "overlap", p, g, m, v, [s[:2], s[2:4]], [s[4:6], s[5:7]])
