"""Norms around a block with gate and residual scale, forward and backward, against the formulas in 64 bits (gradients by differentiation there, and
the differentiated formulas against central differences)."""
import ctypes

import numpy as np
import pytest
import torch

U = 2.0 ** -24


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


def hat(v, layer, eps):
    mean = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    inv = 1 / ((v - mean).square().mean(1, keepdim=True) + eps).sqrt()
    return (v - mean) * inv, mean, inv


def formula(t, layer, eps):
    """y, n and the sizes of what is added up in them, in the tensors' type"""
    y, size = t["x"], t["x"].abs()
    if t["f"] is not None:
        h, mean, inv = hat(t["f"], layer, eps) if t["w_post"] is not None else (t["f"], 0, 1)
        hs = (t["f"].abs() + abs(mean)) * inv
        g = 1 if t["gate"] is None else t["gate"].repeat_interleave(y.shape[0] // t["gate"].shape[0], 0)
        w = 1 if t["w_post"] is None else t["w_post"]
        s = 1 if t["scale"] is None else t["scale"]
        y, size = s * y + g * (w * h), abs(s) * size + abs(g) * abs(w) * hs
    n = nsize = None
    if t["w_pre"] is not None:
        h, mean, inv = hat(y, layer, eps)
        n, nsize = t["w_pre"] * h, t["w_pre"].abs() * (size + abs(mean)) * inv
    return y, n, size, nsize


def inputs(rows, d, bf16, groups, parts, seed=0, spread=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    dt = torch.bfloat16 if bf16 else torch.float32
    row = torch.exp(spread * rnd(rows, 1))
    t = {"x": (rnd(rows, d) * row + shift).to(dt), "f": (rnd(rows, d) * 0.5).to(dt) if "f" in parts else None,
         "w_pre": (1 + 0.1 * rnd(d)).float() if "pre" in parts else None, "w_post": (1 + 0.1 * rnd(d)).float() if "post" in parts else None,
         "gate": (0.5 + 0.2 * rnd(groups, d)).float() if groups else None, "scale": (1 + 0.1 * rnd(d)).float() if "scale" in parts else None}
    t["dy"] = rnd(rows, d).to(dt)
    t["dn"] = rnd(rows, d).to(dt) if "pre" in parts else None
    return t


def gpu(t):
    return {k: None if v is None else v.cuda() for k, v in t.items()}


NAMES = ("x", "w_pre", "f", "w_post", "gate", "scale")
ALL = ("f", "pre", "post", "scale")
CASES = [
    # rows, d, groups, parts
    (1, 1, 0, ("pre",)), (3, 8, 0, ("pre",)), (5, 33, 0, ("f", "pre")), (1, 256, 1, ALL), (7, 257, 7, ALL), (64, 1000, 4, ALL),
    (300, 512, 1, ALL), (300, 520, 300, ("f", "post")), (999, 1001, 1, ALL), (1200, 64, 2, ALL), (130, 4096, 26, ALL), (37, 4104, 0, ALL),
    (40, 8192, 2, ALL), (9, 8200, 0, ("f", "pre", "post")), (5, 16384, 1, ALL), (6, 16383, 2, ALL), (2000, 96, 1000, ("f", "pre", "scale")),
    (450, 128, 3, ("f", "scale")),
]


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,d,groups,parts", CASES)
def test_forward(rows, d, groups, parts, bf16, layer):
    b = sb()
    t = inputs(rows, d, bf16, groups, parts, seed=d)
    c = gpu(t)
    eps = 1e-5
    y, n, stats = b.norm_forward(*[c[k] for k in NAMES], kind=b.SB_NORM_LAYER if layer else b.SB_NORM_RMS, eps=eps, save=True)
    ry, rn, ysize, nsize = formula({k: None if v is None else v.double() for k, v in c.items()}, layer, eps)
    out = 2.0 ** -8 if bf16 else U
    # a row's mean or sum of squares: log2(d) + 8 roundings of the tree of sums, of what is added; a dozen more for the rest
    k = (np.log2(d) + 24) * U
    assert ((y.double() - ry).abs() <= (out * ry.abs() + k * ysize) * 1.01).all()
    if n is not None:
        assert ((n.double() - rn).abs() <= (out * rn.abs() + 2 * k * nsize) * 1.01).all()
    y2, n2 = b.norm_forward(*[c[k] for k in NAMES], kind=b.SB_NORM_LAYER if layer else b.SB_NORM_RMS, eps=eps)
    assert torch.equal(y, y2) and (n is None or torch.equal(n, n2))


def gradients(t, layer, eps):
    leaves = [k for k in NAMES if t[k] is not None]
    a = {k: None if v is None else (v.double().requires_grad_() if k in leaves else v.double()) for k, v in t.items()}
    y, n, _, _ = formula(a, layer, eps)
    loss = (0 if a["dy"] is None else (y * a["dy"]).sum()) + (0 if a["dn"] is None else (n * a["dn"]).sum())
    return dict(zip(leaves, torch.autograd.grad(loss, [a[k] for k in leaves], allow_unused=True)))


TO = {"x": "dx", "w_pre": "dw_pre", "f": "df", "w_post": "dw_post", "gate": "dgate", "scale": "dscale"}


def sizes_of_gradients(t, layer, eps):
    """what is added up in each gradient, taken positive"""
    t = {k: None if v is None else v.double() for k, v in t.items()}
    R = t["x"].shape[0]
    y, _, ysize, _ = formula(t, layer, eps)
    d = torch.zeros_like(y) if t["dy"] is None else t["dy"].abs()
    s = {}
    if t["dn"] is not None:
        h, mean, inv = hat(y, layer, eps)
        hs = (ysize + mean.abs()) * inv
        z = (t["dn"] * t["w_pre"]).abs()
        d = d + inv * (z + hs * (z * hs).mean(1, keepdim=True) + z.mean(1, keepdim=True))
        s["w_pre"] = (t["dn"].abs() * hs).sum(0)
    sc = 1 if t["scale"] is None else t["scale"].abs()
    s["x"] = sc * d
    s["scale"] = (d * t["x"].abs()).sum(0)
    if t["f"] is not None:
        h, mean, inv = hat(t["f"], layer, eps) if t["w_post"] is not None else (t["f"], torch.zeros(1), 1)
        hs = (t["f"].abs() + mean.abs().to(t["f"].device)) * inv
        g = 1 if t["gate"] is None else t["gate"].abs().repeat_interleave(R // t["gate"].shape[0], 0)
        w = 1 if t["w_post"] is None else t["w_post"].abs()
        s["w_post"] = (g * d * hs).sum(0)
        q = g * w * d
        s["f"] = inv * (q + hs * (q * hs).mean(1, keepdim=True) + q.mean(1, keepdim=True)) if t["w_post"] is not None else q
        if t["gate"] is not None:
            s["gate"] = (d * w * hs).view(t["gate"].shape[0], -1, y.shape[1]).sum(1)
    return s


def check_backward(b, t, layer, eps=1e-5, drop=()):
    c = gpu(t)
    bf16 = t["x"].dtype == torch.bfloat16
    kind = b.SB_NORM_LAYER if layer else b.SB_NORM_RMS
    stats = b.norm_forward(*[c[k] for k in NAMES], kind=kind, eps=eps, save=True)[2]
    for k in drop:
        c[k] = None
    got = b.norm_backward(c["dy"], c["dn"], stats, *[c[k] for k in NAMES], kind=kind)
    again = b.norm_backward(c["dy"], c["dn"], stats, *[c[k] for k in NAMES], kind=kind)
    ref, size = gradients(c, layer, eps), sizes_of_gradients(c, layer, eps)
    R, d = t["x"].shape
    for k in NAMES:
        if c[k] is None or (k == "w_pre" and c["dn"] is None):
            assert got[TO[k]] is None
            continue
        r = torch.zeros_like(c[k], dtype=torch.float64) if ref[k] is None else ref[k]
        out = 2.0 ** -8 if bf16 and k in ("x", "f") else U
        # a row's sums as in the forward pass, each mean entering twice over (through the hats); a vector's sum over the rows, one after the other within
        # a CTA and then over these: at most rows / 4 + 200 roundings of what is added in the longest chain
        roundings = 6 * (np.log2(d) + 24) + (0 if k in ("x", "f") else min(R, R / 4 + 200))
        bound = (out * r.abs() + roundings * U * size[k]) * 1.01 + 1e-30
        worst = ((got[TO[k]].double() - r).abs() / bound).max().item()
        assert worst <= 1, (k, worst)
        assert torch.equal(got[TO[k]], again[TO[k]])


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,d,groups,parts", CASES)
def test_backward(rows, d, groups, parts, bf16, layer):
    check_backward(sb(), inputs(rows, d, bf16, groups, parts, seed=d + 1), layer)


@pytest.mark.gpu
@pytest.mark.parametrize("drop", [("dy",), ("dn",)])
def test_backward_of_one_output(drop):
    check_backward(sb(), inputs(50, 264, True, 5, ALL), True, drop=drop)


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [False, True])
def test_rows_that_are_zero_large_or_not_finite(layer):
    """Rows of zeros and of one value, rows near the largest floats' square root, and rows that are not finite: each spoils itself alone."""
    b = sb()
    t = inputs(12, 128, False, 0, ("pre",))
    t["x"][1], t["x"][2], t["x"][3] = 0, 5.0, t["x"][3] * 1e15
    clean = gpu(t)
    t["x"][4, 7], t["x"][5, 9] = float("nan"), float("inf")
    c = gpu(t)
    kind = b.SB_NORM_LAYER if layer else b.SB_NORM_RMS
    n, m = b.norm_forward(c["x"], c["w_pre"], kind=kind)[1], b.norm_forward(clean["x"], clean["w_pre"], kind=kind)[1]
    keep = [i for i in range(12) if i not in (4, 5)]
    assert torch.equal(n[keep], m[keep]) and torch.isfinite(m).all()
    assert (m[1] == 0).all() and torch.isnan(n[4]).all() and torch.isnan(n[5, 9])
    if layer:
        assert (m[2].abs() <= 1e-2).all()


def test_formula_against_differences():
    t = {k: None if v is None else v.double() for k, v in inputs(6, 10, False, 3, ALL, spread=0.2).items()}
    for layer in (False, True):
        g = gradients(t, layer, 1e-5)
        for k in NAMES:
            v = torch.randn(t[k].shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
            f = []
            for e in (1e-5, -1e-5):
                y, n, _, _ = formula({**t, k: t[k] + e * v}, layer, 1e-5)
                f.append(((y * t["dy"]).sum() + (n * t["dn"]).sum()).item())
            # (third derivatives times 1e-10, and 64-bit roundings of sums of some hundred over 2e-5)
            assert abs((f[0] - f[1]) / 2e-5 - (g[k] * v).sum().item()) <= 1e-6


@pytest.mark.gpu
def test_no_rows_and_other_streams():
    b = sb()
    t = gpu(inputs(48, 96, True, 6, ALL))
    e = gpu(inputs(0, 96, True, 0, ("f", "pre", "post")))
    y, n, st = b.norm_forward(*[e[k] for k in NAMES], save=True)
    assert y.shape == (0, 96) and n.shape == (0, 96)
    out = b.norm_backward(e["dy"], e["dn"], st, *[e[k] for k in NAMES])
    assert (out["dw_pre"] == 0).all() and (out["dw_post"] == 0).all()
    ref = b.norm_forward(*[t[k] for k in NAMES], save=True)
    back = b.norm_backward(t["dy"], t["dn"], ref[2], *[t[k] for k in NAMES])
    # two at once, and captured and replayed on changed inputs
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(b.norm_backward(t["dy"], t["dn"], ref[2], *[t[k] for k in NAMES]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd = b.norm_forward(*[t[k] for k in NAMES], save=True)
        bwd = b.norm_backward(t["dy"], t["dn"], fwd[2], *[t[k] for k in NAMES])
    keep = t["x"].clone()
    t["x"].zero_()
    graph.replay()
    t["x"].copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    for other in got + [bwd]:
        for k, v in back.items():
            assert torch.equal(v, other[k]), k
    for a, c in zip(ref, fwd):
        assert torch.equal(a, c)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 100, 4096])
def test_addresses_that_are_not_aligned(d):
    """Matrices and vectors one element behind an aligned address: the same values as at aligned ones, up to the order of the sums."""
    b = sb()
    for bf16 in (False, True):
        t = gpu(inputs(40, d, bf16, 4, ALL))
        off = {k: None if v is None else torch.cat([v.new_zeros(1), v.reshape(-1)])[1:].view(v.shape) for k, v in t.items()}
        st, so = (b.norm_forward(*[c[k] for k in NAMES], save=True) for c in (t, off))
        u = 2.0 ** -7 if bf16 else 2.0 ** -18          # a step of the result's type where a sum in another order falls to the other side; float: the sums' own bound
        for p, q in zip(st[:2], so[:2]):
            assert ((p.double() - q.double()).abs() <= u * (p.double().abs() + p.double().abs().mean())).all()
        back, boff = b.norm_backward(t["dy"], t["dn"], st[2], *[t[k] for k in NAMES]), b.norm_backward(off["dy"], off["dn"], st[2], *[off[k] for k in NAMES])
        for k, p in back.items():
            tol = u if k in ("dx", "df") else 2.0 ** -18
            assert ((p.double() - boff[k].double()).abs() <= tol * (p.double().abs() + 4 * p.double().abs().mean())).all(), k


@pytest.mark.gpu
def test_more_than_2_32_elements():
    """Rows behind the 2^32nd element: the same bits as by themselves (a row's arithmetic does not depend on the number of rows)."""
    b = sb()
    rows, d, some = (1 << 32) // 1024 + 5000, 1024, 3000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
    x[:some].normal_(generator=g)
    x[some:-some] = 0.5
    x[-some:].normal_(generator=g)
    w = torch.rand(d, generator=g, device="cuda")
    _, n, st = b.norm_forward(x, w, save=True)
    for part in (slice(0, some), slice(rows - some, rows)):
        _, m, s2 = b.norm_forward(x[part].clone(), w, save=True)
        assert torch.equal(n[part], m) and torch.equal(st[part], s2)
    dx = b.norm_backward(None, x, st, x, w)["dx"]
    m = b.norm_backward(None, x[-some:].clone(), st[-some:].clone(), x[-some:].clone(), w)["dx"]
    assert torch.equal(dx[-some:], m)


def test_refusals():
    b = sb()
    a, n = ctypes.c_void_p(0x1000), None
    ok = dict(rows=4, groups=2, d=8, kind=0, precision=1, eps=1e-6)
    cfg = lambda **k: b.sb_norm_config(*[{**ok, **k}[x] for x in ("rows", "groups", "d", "kind", "precision", "eps")])  # noqa: E731
    fwd = lambda c, *p: b.sb_norm_forward(ctypes.byref(c), *p, n)  # noqa: E731
    every = (a,) * 9          # x, w_pre, f, w_post, gate, scale, y, n, stats
    for bad, status in ((dict(kind=2), 1), (dict(precision=3), 1), (dict(rows=-1), 2), (dict(d=0), 2), (dict(d=16385), 3), (dict(groups=3), 2),
                        (dict(groups=-1), 2), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1)):
        assert fwd(cfg(**bad), *every) == status, bad
        size = ctypes.c_size_t()
        assert b.sb_norm_bytes(ctypes.byref(cfg(**bad)), ctypes.byref(size)) == status
    assert b.sb_norm_forward(None, *every, n) == 1
    for i, status in ((0, 1), (1, 1), (2, 1), (4, 1), (7, 1)):       # one pointer missing: x, w_pre (n is there), f (its vectors are), gate, n
        p = list(every)
        p[i] = n
        assert fwd(cfg(), *p) == status, i
    assert fwd(cfg(groups=0), *every) == 1
    assert fwd(cfg(groups=0), a, n, n, n, n, n, n, n, n) == 1
    assert fwd(cfg(), ctypes.c_void_p(0x1001), *every[1:]) == 1
    bwd = lambda c, p, ws=a, size=1 << 20: b.sb_norm_backward(ctypes.byref(c), *p, ws, size, n)  # noqa: E731
    every = (a,) * 15         # dy, dn, stats, x, w_pre, f, w_post, gate, scale, dx, df, dw_pre, dw_post, dgate, dscale
    for missing in ((0, 1), (4,), (2,), (3,), (5,), (6,), (7,), (8,), (1,)):
        p = [n if i in missing else v for i, v in enumerate(every)]
        assert bwd(cfg(), p) == 1, missing
    assert bwd(cfg(), every, n) == 4 and bwd(cfg(), every, a, 16) == 4 and bwd(cfg(), every, ctypes.c_void_p(0x1004)) == 4
    assert "workspace" in b.sb_last_error()
    x = torch.zeros(4, 8)
    with pytest.raises(b.SBError):
        b.norm_forward(x, torch.ones(8))


@pytest.mark.gpu
def test_binding_refusals():
    b = sb()
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    for bad in (dict(w_pre=w.double()), dict(w_pre=w[:4]), dict(w_pre=w, f=x.t().contiguous().t()), dict(w_pre=w, f=x.bfloat16()), dict(w_pre=w.cpu()),
                dict(w_pre=w, f=x, gate=torch.ones(3, 8, device="cuda"))):
        with pytest.raises(b.SBError):
            b.norm_forward(x, **bad)
    for bad in (x.half(), x[:, ::2], x[0]):
        with pytest.raises(b.SBError):
            b.norm_forward(bad, w)


def test_misaligned_vectors_are_refused():
    """Vectors and their gradients are floats: any other address would be a fault of the kernel's."""
    b = sb()
    a, odd, n = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002), None
    c = ctypes.byref(b.sb_norm_config(4, 2, 8, 0, 1, 1e-6))
    for i in (1, 3, 4, 5):                    # w_pre, w_post, gate, scale
        assert b.sb_norm_forward(c, *[odd if k == i else a for k in range(9)], n) == 1, i
        assert "misaligned" in b.sb_last_error()
    for i in (4, 6, 7, 8, 11, 12, 13, 14):    # the same, and their gradients
        assert b.sb_norm_backward(c, *[odd if k == i else a for k in range(15)], a, 1 << 20, n) == 1, i
        assert "misaligned" in b.sb_last_error()
