"""AdamW with float moments: root and quotient of a parameter's step are rounded as float operations are.  From parameters of zero and without eps every
operation of the step has one rounding only (a fused multiply-add with a zero rounds like the product), so that numpy's floats give the same bits."""
import numpy as np
import pytest


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n", [1, 1000, 300001])
def test_step_is_rounded_as_float_operations_are(n, bf16):
    import torch
    b, f = sb(), np.float32
    g = torch.Generator().manual_seed(n)
    rnd = lambda: torch.randn(n, generator=g)  # noqa: E731
    p, m, v = torch.zeros(n, device="cuda"), (rnd() * 1e-3).cuda(), (torch.exp(4 * rnd()) * 1e-6).cuda()
    grad = (rnd() * 1e-2).to(torch.bfloat16 if bf16 else torch.float32).cuda()
    lr, b1, b2, t = 1e-2, 0.9, 0.99, 3
    b.AdamW([p], [grad], [m], [v]).step(lr, beta1=b1, beta2=b2, eps=0.0, weight_decay=0.1, step=t)
    m, v = m.cpu().numpy(), v.cpu().numpy()
    assert (v > 0).all()
    rate, rs2 = f(lr / (1 - b1 ** t)), f(1 / np.sqrt(1 - b2 ** t))
    step = rate * (m / (np.sqrt(v) * rs2))
    assert step.dtype == np.float32
    assert np.array_equal(p.cpu().numpy(), -step)
