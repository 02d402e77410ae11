"""Gated feed-forward block, forward and backward, against the formulas in 64 bits, with bounds for every element from the roundings that are made."""
import ctypes

import pytest
import torch

U = 2.0 ** -24


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


ACTS = ("silu", "gelu", "relu")


def act_of(g, name):
    """a(g), a'(g)"""
    if name == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    cdf = 0.5 * torch.erfc(-g / 2 ** 0.5)
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / (2 * torch.pi) ** 0.5


def inputs(rows, d, f, bf16, seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    dt = torch.bfloat16 if bf16 else torch.float32
    return [t.to(dt).cuda() for t in (rnd(rows, d), rnd(2 * f, d) / d ** 0.5, rnd(d, f) / f ** 0.5, rnd(rows, d))]


# What a sum of K products may be off, relative to the sum of their magnitudes: float sums of exact bf16 products, in tiles and then over these;
# float operands as three bf16 terms each leave out products of 2^-24 of the largest, on top of the roundings of the sums
def sum_error(k):
    return (k + 32) * U


# a(g) and a'(g) by the approximations of exp and division: a few units in the last place of a float; 2^-21 is granted
ACT = 2.0 ** -21


def check_forward(b, rows, d, f, bf16, act, seed=0):
    x, wgu, wd, _ = inputs(rows, d, f, bf16, seed)
    kind = {"silu": b.SB_ACT_SILU, "gelu": b.SB_ACT_GELU, "relu": b.SB_ACT_RELU}[act]
    y, gu = b.ffn_forward(x, wgu, wd, kind, save=True)
    b.ops_check()
    X, W, D = x.double(), wgu.double(), wd.double()
    out = 2.0 ** -8 if bf16 else U
    ref = X @ W.t()
    gerr = sum_error(d) * (X.abs() @ W.abs().t())
    assert ((gu.double() - ref).abs() <= (out * ref.abs() + gerr) * 1.01).all()
    a, da = act_of(ref[:, :f], act)
    h = a * ref[:, f:]
    # |a'| is at most 1.13 for all three
    herr = 1.13 * gerr[:, :f] * ref[:, f:].abs() + a.abs() * gerr[:, f:] + 1.13 * gerr[:, :f] * gerr[:, f:] + (ACT + out) * h.abs() + ACT * ref[:, f:].abs() * 2.0 ** -3
    yref = h @ D.t()
    bound = out * yref.abs() + sum_error(f) * (h.abs() @ D.abs().t()) + herr @ D.abs().t()
    worst = ((y.double() - yref).abs() / (bound * 1.01 + 1e-30)).max().item()
    assert worst <= 1, worst
    assert torch.equal(y, b.ffn_forward(x, wgu, wd, kind))          # (nothing kept: the same bits)
    return y, gu


def check_backward(b, rows, d, f, bf16, act, grad_f32=False, seed=0):
    x, wgu, wd, dy = inputs(rows, d, f, bf16, seed)
    kind = {"silu": b.SB_ACT_SILU, "gelu": b.SB_ACT_GELU, "relu": b.SB_ACT_RELU}[act]
    gu = (x.float() @ wgu.float().t()).to(x.dtype)
    got = b.ffn_backward(dy, x, gu, wgu, wd, kind, grad_dtype=torch.float32 if grad_f32 else None)
    b.ops_check()
    X, W, D, dY, G, Uv = x.double(), wgu.double(), wd.double(), dy.double(), gu[:, :f].double(), gu[:, f:].double()
    out = 2.0 ** -8 if bf16 else U
    a, da = act_of(G, act)
    dh = dY @ D
    dherr = sum_error(d) * (dY.abs() @ D.abs())
    dgu = torch.cat([dh * Uv * da, dh * a], 1)
    err = torch.cat([dherr * (Uv * da).abs() + ACT * (dh.abs() + dherr) * Uv.abs(), dherr * a.abs() + ACT * (dh.abs() + dherr) * (a.abs() + G.abs() * 2.0 ** -3)], 1) + out * dgu.abs() * 1.01
    h = a * Uv
    herr = (out + ACT) * h.abs() + ACT * 2.0 ** -3 * (G * Uv).abs()
    wout = 2.0 ** -8 if bf16 and not grad_f32 else U
    for name, t, ref, bound in (
            ("dx", got[0], dgu @ W, out * (dgu @ W).abs() + sum_error(2 * f) * (dgu.abs() @ W.abs()) + err @ W.abs()),
            ("dw_gate_up", got[1], dgu.t() @ X, wout * (dgu.t() @ X).abs() + sum_error(rows) * (dgu.abs().t() @ X.abs()) + err.t() @ X.abs()),
            ("dw_down", got[2], dY.t() @ h, wout * (dY.t() @ h).abs() + sum_error(rows) * (dY.abs().t() @ h.abs()) + dY.abs().t() @ herr)):
        worst = ((t.double() - ref).abs() / (bound * 1.01 + 1e-30)).max().item()
        assert worst <= 1, (name, worst)
    again = b.ffn_backward(dy, x, gu, wgu, wd, kind, grad_dtype=torch.float32 if grad_f32 else None)
    assert all(torch.equal(p, q) for p, q in zip(got, again))
    only = b.ffn_backward(dy, x, gu, wgu, wd, kind, grad_dtype=torch.float32 if grad_f32 else None, needs=(False, False, True))
    assert only[0] is None and only[1] is None and torch.equal(only[2], got[2])


ROWS = [1, 2, 7, 8, 16, 17, 33, 64, 65, 111, 128, 129, 200, 256, 257, 300, 512, 640, 1025]
WIDTHS = [(64, 64), (72, 40), (136, 1368), (256, 512), (520, 264)]


@pytest.mark.gpu
@pytest.mark.parametrize("d,f", WIDTHS)
@pytest.mark.parametrize("rows", ROWS)
def test_forward_bf16(rows, d, f):
    check_forward(sb(), rows, d, f, True, ACTS[rows % 3], seed=rows)


@pytest.mark.gpu
@pytest.mark.parametrize("d,f", WIDTHS)
@pytest.mark.parametrize("rows", ROWS)
def test_backward_bf16(rows, d, f):
    check_backward(sb(), rows, d, f, True, ACTS[rows % 3], grad_f32=rows % 2 == 0, seed=rows)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d,f", [(1, 1, 1), (3, 33, 17), (130, 129, 65), (40, 30, 132), (257, 70, 31)])
@pytest.mark.parametrize("bf16", [False, True])
def test_any_width(rows, d, f, bf16):
    for act in ACTS:
        check_forward(sb(), rows, d, f, bf16, act)
        check_backward(sb(), rows, d, f, bf16, act, grad_f32=act == "relu")


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d,f", [(1, 64, 128), (64, 136, 264), (300, 256, 512), (1000, 512, 264)])
def test_float(rows, d, f):
    check_forward(sb(), rows, d, f, False, ACTS[rows % 3])
    check_backward(sb(), rows, d, f, False, ACTS[rows % 3])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d,f", [(1, 4096, 8192), (5, 4096, 1024), (48, 1024, 4096), (1100, 4096, 1032), (2500, 1032, 2056)])
def test_large(rows, d, f):
    check_forward(sb(), rows, d, f, True, ACTS[rows % 3])
    check_backward(sb(), rows, d, f, True, ACTS[rows % 3])


@pytest.mark.gpu
def test_gradients_against_differences():
    """Float gradients against central differences of the formula in 64 bits, along a random direction in each operand.  The difference itself is off by
    third derivatives times 1e-10 and 64-bit roundings over 2e-5; the gradient by the bounds of the tests above, 1e-6 of the sums of magnitudes."""
    b = sb()
    rows, d, f = 20, 24, 40
    for act, kind in zip(ACTS, (b.SB_ACT_SILU, b.SB_ACT_GELU, b.SB_ACT_RELU)):
        x, wgu, wd, dy = inputs(rows, d, f, False, 5)
        _, gu = b.ffn_forward(x, wgu, wd, kind, save=True)
        grads = b.ffn_backward(dy, x, gu, wgu, wd, kind)

        def loss(x, wgu, wd):
            gu = x @ wgu.t()
            return (((act_of(gu[:, :f], act)[0] * gu[:, f:]) @ wd.t()) * dy.double()).sum().item()

        args = [t.double() for t in (x, wgu, wd)]
        for k in range(3):
            v = torch.randn(args[k].shape, generator=torch.Generator().manual_seed(k), dtype=torch.float64).cuda()
            hi, lo = (loss(*[a + (e * v if i == k else 0) for i, a in enumerate(args)]) for e in (1e-5, -1e-5))
            size = (grads[k].double().abs() * v.abs()).sum().item()
            assert abs((hi - lo) / 2e-5 - (grads[k].double() * v).sum().item()) <= 2e-5 * size


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 100, 400])
def test_rows_stand_alone(rows):
    """A row that is not finite spoils its own outputs only; other rows keep their bits, whatever their number; extreme values of the activation."""
    b = sb()
    x, wgu, wd, dy = inputs(rows, 136, 264, True, 9)
    x[0] *= 100
    y = b.ffn_forward(x, wgu, wd)
    bad = x.clone()
    bad[1, 5], bad[rows - 1, 7] = float("nan"), float("inf")
    z = b.ffn_forward(bad, wgu, wd)
    keep = [i for i in range(rows) if i not in (1, rows - 1)]
    assert torch.equal(y[keep], z[keep]) and torch.isfinite(y).all()
    assert torch.isnan(z[1]).all() and not torch.isfinite(z[rows - 1]).any()
    # a gate far below zero: silu and gelu are zero there, not NaN
    for kind in (b.SB_ACT_SILU, b.SB_ACT_GELU):
        low = torch.full((rows, 64), -200.0, dtype=torch.bfloat16, device="cuda")
        w = torch.ones(128, 64, dtype=torch.bfloat16, device="cuda")
        out, gu = b.ffn_forward(low, w, torch.ones(64, 64, dtype=torch.bfloat16, device="cuda"), kind, save=True)
        assert (out == 0).all()
        dx, dwgu, dwd = b.ffn_backward(low, low, gu, w, torch.ones(64, 64, dtype=torch.bfloat16, device="cuda"), kind)
        assert (dx == 0).all() and (dwgu == 0).all() and (dwd == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [4, 90, 600])
@pytest.mark.parametrize("bf16", [True, False])
def test_streams_and_graphs(rows, bf16):
    b = sb()
    x, wgu, wd, dy = inputs(rows, 256, 264, bf16, 3)
    y, gu = b.ffn_forward(x, wgu, wd, save=True)
    grads = b.ffn_backward(dy, x, gu, wgu, wd)
    torch.cuda.synchronize()
    got = []
    for s in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(s):
            got.append((b.ffn_forward(x, wgu, wd, save=True), b.ffn_backward(dy, x, gu, wgu, wd)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd = b.ffn_forward(x, wgu, wd, save=True)
        bwd = b.ffn_backward(dy, x, fwd[1], wgu, wd)
    keep = x.clone()
    x.zero_()
    graph.replay()
    x.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    for (f2, b2) in got + [(fwd, bwd)]:
        assert torch.equal(y, f2[0]) and torch.equal(gu, f2[1])
        assert all(torch.equal(p, q) for p, q in zip(grads, b2))
    b.ops_check()


@pytest.mark.gpu
def test_more_than_2_32_elements():
    """GU of more than 2^32 elements: the last rows as in a call of their own (the same kernel, whose rows do not depend on one another)."""
    b = sb()
    d, f, some = 64, 2048, 70000
    rows = (1 << 32) // (2 * f) + some
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    x[-some:] = rnd(some, d)
    wgu, wd = rnd(2 * f, d), rnd(d, f)
    y, gu = b.ffn_forward(x, wgu, wd, save=True)
    y2, gu2 = b.ffn_forward(x[-some:].clone(), wgu, wd, save=True)
    assert torch.equal(y[-some:], y2) and torch.equal(gu[-some:], gu2)
    dx = b.ffn_backward(x, x, gu, wgu, wd, needs=(True, False, False))[0]
    dx2 = b.ffn_backward(x[-some:].clone(), x[-some:].clone(), gu2, wgu, wd, needs=(True, False, False))[0]
    assert torch.equal(dx[-some:], dx2)
    b.ops_check()


@pytest.mark.gpu
def test_no_rows():
    b = sb()
    x, wgu, wd, dy = inputs(0, 64, 128, True)
    y, gu = b.ffn_forward(x, wgu, wd, save=True)
    assert y.shape == (0, 64) and gu.shape == (0, 256)
    dx, dwgu, dwd = b.ffn_backward(dy, x, gu, wgu, wd)
    assert dx.shape == (0, 64) and (dwgu == 0).all() and (dwd == 0).all()


def test_refusals():
    b = sb()
    a, n = ctypes.c_void_p(0x1000), None
    ok = dict(rows=4, d=8, f=16, act=0, precision=1, grad=0)
    cfg = lambda **k: b.sb_ffn_config(*[{**ok, **k}[x] for x in ("rows", "d", "f", "act", "precision", "grad")])  # noqa: E731
    size = ctypes.c_size_t()
    for bad, status in ((dict(rows=-1), 2), (dict(d=0), 2), (dict(f=0), 2), (dict(act=3), 1), (dict(act=-1), 1), (dict(precision=2), 1), (dict(grad=2), 1),
                        (dict(precision=0, grad=1), 1), (dict(rows=2 ** 31), 3), (dict(f=2 ** 20 + 1), 3), (dict(d=2 ** 20 + 1), 3)):
        assert b.sb_ffn_bytes(ctypes.byref(cfg(**bad)), 0, ctypes.byref(size)) == status, bad
        assert b.sb_ffn_forward(ctypes.byref(cfg(**bad)), a, a, a, a, a, a, 1 << 40, n) == status, bad
        assert b.sb_ffn_backward(ctypes.byref(cfg(**bad)), a, a, a, a, a, a, a, a, a, 1 << 40, n) == status, bad
    assert b.sb_ffn_bytes(None, 0, ctypes.byref(size)) == 1 and b.sb_ffn_bytes(ctypes.byref(cfg()), 0, None) == 1
    fwd = lambda p, ws=a, bytes_=1 << 30: b.sb_ffn_forward(ctypes.byref(cfg()), *p, ws, bytes_, n)  # noqa: E731
    every = [a] * 5           # x, w_gate_up, w_down, gu, y
    for i in range(5):
        assert i == 3 or fwd([n if k == i else v for k, v in enumerate(every)]) == 1
        assert fwd([ctypes.c_void_p(0x1008) if k == i else v for k, v in enumerate(every)]) == 1
    assert fwd(every, n) == 1 and fwd(every, ctypes.c_void_p(0x1010)) == 1 and fwd(every, a, 16) == 4
    assert "workspace" in b.sb_last_error()
    bwd = lambda p, ws=a, bytes_=1 << 30: b.sb_ffn_backward(ctypes.byref(cfg()), *p, ws, bytes_, n)  # noqa: E731
    every = [a] * 8           # dy, x, gu, w_gate_up, w_down, dx, dw_gate_up, dw_down
    for i in range(8):
        assert i >= 5 or bwd([n if k == i else v for k, v in enumerate(every)]) == 1
        assert bwd([ctypes.c_void_p(0x1008) if k == i else v for k, v in enumerate(every)]) == 1
    assert bwd(every, n) == 1 and bwd(every, a, 16) == 4
    x = torch.zeros(4, 8)
    with pytest.raises(b.SBError):
        b.ffn_forward(x, torch.zeros(16, 8), torch.zeros(8, 8))


@pytest.mark.gpu
def test_binding_refusals():
    b = sb()
    x, wgu, wd, dy = inputs(4, 64, 32, True)
    gu = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in ((x.half(), wgu, wd), (x, wgu.float(), wd), (x, wgu[:-1], wd), (x, wgu, wd.t()), (x[:, ::2], wgu, wd), (x, wgu.cpu(), wd), (x[0], wgu, wd)):
        with pytest.raises(b.SBError):
            b.ffn_forward(*bad)
    for bad in ((dy.float(), x, gu), (dy, x, gu[:, :32]), (dy[:2], x, gu)):
        with pytest.raises(b.SBError):
            b.ffn_backward(*bad, wgu, wd)
    with pytest.raises(b.SBError):
        b.ffn_backward(dy, x, gu, wgu, wd, grad_dtype=torch.float16)
    odd = torch.zeros(5 * 33 + 1, device="cuda")[1:].view(5, 33)          # not 16-byte aligned
    with pytest.raises(b.SBError):
        b.ffn_forward(odd, torch.zeros(34, 33, device="cuda"), torch.zeros(33, 17, device="cuda"))
