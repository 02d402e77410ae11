"""AdamW over lists of tensors: float moments against the formulas in 64 bits, 8-bit moments bit for bit against a numpy restatement of the
codes (powers of two as scales, e4m3 to nearest even, five bits of exponent and three of mantissa rounded by given random bits)."""
import numpy as np
import pytest

U = 2.0 ** -24          # half a step of a float, relative


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


# ---- the codes in numpy ----------------------------------------------------------------------------------------------


def philox_halves(n, seed, tensor, step):
    from oracle.splitbrain_oracle import philox4x32_10
    e = np.arange((n + 7) // 8, dtype=np.uint64)
    words = philox4x32_10(e & np.uint64(0xFFFFFFFF), e >> np.uint64(32), tensor, step & 0xFFFFFFFF, seed & 0xFFFFFFFF, seed >> 32)
    return np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in words for s in (0, 16)], 1).astype(np.uint32).reshape(-1)[:n]


def powers(a):
    top = np.where(np.isfinite(a), np.abs(a), 0).max(1).astype(np.float32)
    top = np.maximum(top, np.float32(2.0 ** -100))
    return (top.view(np.uint32) & 0x7F800000).view(np.float32)


def blocks(a):
    out = np.zeros((-(-a.size // 256), 256), a.dtype)
    out.reshape(-1)[:a.size] = a
    return out


def e4m3_value(code):
    code = code.astype(np.int64)
    e, m, sign = (code >> 3) & 15, code & 7, np.where(code & 128, -1.0, 1.0)
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    return np.where((code & 127) == 127, np.nan, sign * v)


def encode_m(m):
    b = blocks(m)
    scale = powers(b) * np.float32(2.0 ** -7)
    q = b.astype(np.float64) / scale[:, None]
    ulp = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(np.where(np.isfinite(q), q, 1)), 2.0 ** -6))) - 3)
    return (np.rint(q / ulp) * ulp).reshape(-1)[:m.size], scale          # (what the codes stand for, in units of the scale)


def encode_v(v, half):
    b = blocks(v)
    scale = powers(b)
    q = b.astype(np.float64) / scale[:, None]
    ulp = 2.0 ** (np.floor(np.log2(np.maximum(np.where(np.isfinite(q), q, 1), 2.0 ** -29))) - 3)
    return (np.floor(q / ulp + blocks(half.astype(np.float64)) / 65536.0) * ulp).reshape(-1)[:v.size], scale


def unit_v(code):
    code = code.astype(np.int64)
    e, f = code >> 3, code & 7
    return np.where(code == 255, np.nan, np.where(e > 0, (1 + f / 8.0) * 2.0 ** (e - 30.0), f / 8.0 * 2.0 ** -29))


def moments32(m, v, g, b1, b2):
    """the moments in float, rounded as the formulas are written"""
    f = np.float32
    return f(b1) * m + f(1.0 - b1) * g, f(b2) * v + (f(1.0 - b2) * g) * g


def reference(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay):
    p, g, m, v = (a.astype(np.float64) for a in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = lr / (1 - beta1 ** t) * m / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return (1 - lr * weight_decay) * p - step, m, v, step


SIZES = [[1], [7], [255, 256, 257], [1000, 3, 64, 8192, 1], [0, 5, 0, 513]]


def tensors(sizes, seed, bf16, offset=0):
    import torch
    rng = np.random.default_rng(seed)
    made = []
    for n in sizes:
        p, m = rng.standard_normal(n).astype(np.float32), (rng.standard_normal(n) * 1e-3).astype(np.float32)
        v = (np.exp(2 * rng.standard_normal(n)) * 1e-6).astype(np.float32)
        g = (rng.standard_normal(n) * np.exp(rng.standard_normal(n)) * 1e-2).astype(np.float32)
        if bf16:
            g = torch.from_numpy(g).to(torch.bfloat16).float().numpy()
        made.append((p, g, m, v))
    return made


def on_gpu(a, dtype=None, offset=0):
    """on the device, `offset` elements behind an aligned address"""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    dtype = dtype or t.dtype
    room = torch.zeros(t.numel() + offset, dtype=dtype, device="cuda")
    room[offset:] = t.to("cuda").to(dtype)
    return room[offset:]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("bf16,offset", [(False, 0), (True, 0), (False, 1), (True, 3)])
def test_float_moments(sizes, bf16, offset):
    import torch
    b, made = sb(), tensors(sizes, 5, bf16)
    p, g, m, v = ([on_gpu(t[k], torch.bfloat16 if bf16 and k == 1 else None, offset) for t in made] for k in range(4))
    shadow = [torch.full_like(x, 7.0, dtype=torch.bfloat16) for x in p]
    opt = b.AdamW(p, g, m, v, shadows=shadow)
    for t in (3, 4):
        before = [tuple(x.cpu().numpy() for x in (p[i], m[i], v[i])) for i in range(len(sizes))]
        opt.step(step=t, **HYPER)
        torch.cuda.synchronize()
        for i, (_, g0, _, _) in enumerate(made):
            p0, m0, v0 = before[i]
            rp, rm, rv, step = reference(p0, g0, m0, v0, t, **HYPER)
            # three roundings a moment (the constants among them); the step: those of m, half those of v, and eight more of its own
            assert np.all(np.abs(m[i].cpu().numpy() - rm) <= 3 * U * (np.abs(0.9 * m0) + np.abs(0.1 * g0.astype(np.float64))))
            assert np.all(np.abs(v[i].cpu().numpy() - rv) <= 5 * U * rv)
            m_err = 3 * U * (np.abs(0.9 * m0) + np.abs(0.1 * g0.astype(np.float64)))
            slope = HYPER["lr"] / (1 - 0.9 ** t) / (np.sqrt(rv / (1 - 0.99 ** t)) + 1e-8)
            bound = 4 * U * (np.abs(p0) + np.abs(step)) + slope * m_err + 12 * U * np.abs(step)
            assert np.all(np.abs(p[i].cpu().numpy() - rp) <= bound)
            assert torch.equal(shadow[i], p[i].to(torch.bfloat16))


def eight_bit_state(made, torch_fp8=True):
    import torch
    m, v, ms, vs = [], [], [], []
    for i, (_, _, m0, v0) in enumerate(made):
        q, s = encode_m(m0)
        table = e4m3_value(np.arange(256))
        order = {x: c for c, x in reversed(list(enumerate(table))) if not np.isnan(x)}
        m.append(torch.from_numpy(np.array([order[x] for x in q], np.uint8)).cuda())
        ms.append(torch.from_numpy(s).cuda())
        q, s = encode_v(v0, np.zeros(v0.size))
        order = {x: c for c, x in enumerate(unit_v(np.arange(255)))}
        v.append(torch.from_numpy(np.array([order[x] for x in q], np.uint8)).cuda())
        vs.append(torch.from_numpy(s).cuda())
    return m, v, ms, vs


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("bf16,offset", [(False, 0), (True, 0), (False, 1)])
def test_eight_bit_moments(sizes, bf16, offset):
    import torch
    b, made = sb(), tensors(sizes, 6, bf16)
    if len(sizes) == 5 and sizes[3] == 8192:          # blocks of zeros, of one element, of magnitudes far apart, the smallest floats
        made[3][1][:256] = 0; made[3][2][:256] = 0; made[3][3][:256] = 0
        made[3][1][256:512] = 0; made[3][2][256:512] = 0; made[3][1][300] = 1e-3
        made[3][1][512:768] *= np.exp2(np.linspace(-40, 20, 256)).astype(np.float32)
        made[3][1][768:1024] = 1e-38; made[3][2][768:1024] = 0; made[3][3][768:1024] = 0
        made[3][1][1024:1280] = 1e15; made[3][2][1024:1280] = 0
        if bf16:
            made[3][1][:] = torch.from_numpy(made[3][1]).to(torch.bfloat16).float().numpy()
    seed = 0x1234567890ABCDEF
    p, g = ([on_gpu(t[k], torch.bfloat16 if bf16 and k == 1 else None, offset) for t in made] for k in range(2))
    m, v, ms, vs = eight_bit_state(made)
    m, v = ([on_gpu(x.cpu().numpy(), None, offset) for x in side] for side in (m, v))
    opt = b.AdamW(p, g, m, v, ms, vs, seed=seed)
    for t in (1, 2, 2 ** 32 + 5):
        before = [[x[i].cpu().numpy() for x in (p, m, v, ms, vs)] for i in range(len(sizes))]
        opt.step(step=t, **HYPER)
        vm, vv = opt.moments()
        torch.cuda.synchronize()
        for i, (_, g0, _, _) in enumerate(made):
            if not sizes[i]:
                continue
            p0, mc, vc, s_m, s_v = before[i]
            q = np.arange(sizes[i]) // 256
            m0, v0 = (e4m3_value(mc) * s_m[q]).astype(np.float32), (unit_v(vc) * s_v[q]).astype(np.float32)
            m1, v1 = moments32(m0, v0, g0, HYPER["beta1"], HYPER["beta2"])
            rm, rms = encode_m(m1)
            rv, rvs = encode_v(v1, philox_halves(sizes[i], seed, i, t))
            assert np.array_equal(ms[i].cpu().numpy(), rms) and np.array_equal(vs[i].cpu().numpy(), rvs)
            assert np.array_equal(e4m3_value(m[i].cpu().numpy()), rm)
            assert np.array_equal(unit_v(v[i].cpu().numpy()), rv)
            assert np.array_equal(vm[i].float().cpu().numpy(), (rm * rms[q]).astype(np.float32))
            assert np.array_equal(vv[i].float().cpu().numpy(), (rv * rvs[q]).astype(np.float32))
            rp, _, _, step = reference(p0, g0, m0, v0, t, **HYPER)
            slope = HYPER["lr"] / (1 - 0.9 ** t) / (np.sqrt(v1.astype(np.float64) / (1 - 0.99 ** t)) + 1e-8)
            bound = 4 * U * (np.abs(p0) + np.abs(step)) + slope * 3 * U * (np.abs(m0) + np.abs(g0)) + 12 * U * np.abs(step)
            assert np.all(np.abs(p[i].cpu().numpy() - rp) <= bound)


@pytest.mark.gpu
def test_moments_that_are_not_finite_stay_where_they_are():
    """A gradient that is not finite spoils its own element; the others of its block keep their scale and their codes."""
    import torch
    b = sb()
    n = 600
    made = tensors([n], 7, False)
    state = eight_bit_state(made)
    results = []
    for spoil in (False, True):
        p, g = on_gpu(made[0][0]), on_gpu(made[0][1])
        m, v, ms, vs = ([x.clone() for x in side] for side in state)
        if spoil:
            g[10], g[300], g[599] = float("nan"), float("inf"), float("-inf")
        else:
            g[10] = g[300] = g[599] = 0.0
            # (nothing of these elements may set the scale in this run either)
            m[0][[10, 300, 599]] = 0; v[0][[10, 300, 599]] = 0
        opt = b.AdamW([p], [g], m, v, ms, vs, seed=3)
        opt.step(step=1, **HYPER)
        vm, vv = opt.moments()
        results.append([t.float().cpu().numpy() for t in (p, vm[0], vv[0], ms[0], vs[0])])
    keep = np.ones(n, bool)
    keep[[10, 300, 599]] = False
    for a, c in zip(results[0][:3], results[1][:3]):
        assert np.array_equal(a[keep], c[keep])
        assert np.isnan(c[~keep]).all() or c is results[1][0]
    assert np.array_equal(results[0][3], results[1][3]) and np.array_equal(results[0][4], results[1][4])
    assert np.isnan(results[1][0][10])
    # the next step decodes what is not a number as such
    assert np.isnan(results[1][1][~keep]).all() and np.isnan(results[1][2][~keep]).all()


@pytest.mark.gpu
def test_second_moment_decays_in_expectation():
    """With a zero gradient v falls by a factor of beta2 a step; rounding to nearest would leave it where it is.  65536 elements of one value:
    their mean after k steps is beta2^k of the start's, off by the chance of the rounding: each step moves an element's v by one of two neighbouring
    codes, at most an eighth apart, so a step's standard deviation is at most a sixteenth and the mean's after 40 steps at most
    sqrt(40) / 16 / 256 = 0.16 %; six of these are allowed."""
    import torch
    b = sb()
    n = 65536
    z = torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.full((n,), 30 << 3, dtype=torch.uint8, device="cuda")
    ms, vs = (torch.ones(n // 256, device="cuda") for _ in range(2))
    opt = b.AdamW([z], [torch.zeros_like(z)], [m], [v], [ms], [vs], seed=11)
    for t in range(1, 41):
        opt.step(step=t, lr=1e-3, beta2=0.999)
    mean = opt.moments()[1][0].double().mean().item()
    assert abs(mean / 0.999 ** 40 - 1) <= 6 * np.sqrt(40) / 16 / 256


@pytest.mark.gpu
@pytest.mark.parametrize("count", [33, 350, 351, 900])
def test_long_lists(count):
    import torch
    b = sb()
    sizes = [(i * 37) % 700 for i in range(count)]
    made = tensors(sizes, 8, False)
    p, g, m, v = ([on_gpu(t[k]) for t in made] for k in range(4))
    b.AdamW(p, g, m, v).step(step=2, **HYPER)
    for i, (p0, g0, m0, v0) in enumerate(made):
        if sizes[i]:
            rp, rm, rv, step = reference(p0, g0, m0, v0, 2, **HYPER)
            assert np.allclose(m[i].cpu().numpy(), rm, rtol=0, atol=3 * U * float(np.max(np.abs(m0) + np.abs(g0))))
            assert np.max(np.abs(p[i].cpu().numpy() - rp) - 8 * U * np.abs(p0)) <= 1e-5 * np.max(np.abs(step))
    # 8-bit states: an element's random bits go by its tensor's place in the whole list
    m, v, ms, vs = eight_bit_state(made)
    opt = b.AdamW(p, g, m, v, ms, vs, seed=9)
    old = [(x.cpu().numpy(), s.cpu().numpy()) for x, s in zip(v, vs)]
    opt.step(step=7, **HYPER)
    for i in (0, 1, count // 2, count - 1):
        if sizes[i]:
            v0 = (unit_v(old[i][0]) * old[i][1][np.arange(sizes[i]) // 256]).astype(np.float32)
            _, v1 = moments32(v0, v0, made[i][1], HYPER["beta1"], HYPER["beta2"])
            assert np.array_equal(unit_v(v[i].cpu().numpy()), encode_v(v1, philox_halves(sizes[i], 9, i, 7))[0])


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_replayed_in_a_graph_with_its_step_in_device_memory(bits):
    import torch
    b = sb()
    made = tensors([700, 64], 9, False)
    runs = []
    for replay in (False, True):
        p, g, m, v = ([on_gpu(t[k]) for t in made] for k in range(4))
        ms = vs = None
        if bits == 8:
            m, v, ms, vs = eight_bit_state(made)
        opt = b.AdamW(p, g, m, v, ms, vs, seed=4)
        if replay:
            step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    opt.step(0.0, dev_step=step, dev_lr=lr)
            for t in range(1, 4):
                step.fill_(t); lr.fill_(0.01 / t)
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
        else:
            for t in range(1, 4):
                opt.step(float(np.float32(0.01 / t)), step=t)
        runs.append([x.float().cpu().numpy() for x in [*p, *m, *v]])
    for a, c in zip(*runs):
        assert np.array_equal(a, c)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_2_32_elements(bits):
    """The end of a tensor of more than 2^32 elements: as in a tensor of its own (8 bits: with a gradient and moments whose codes need no rounding, since the
    random bits go by the element's place)."""
    import torch
    b = sb()
    n, tail = (1 << 32) + 700, 600 + 256          # (from a block's first element)
    lo = n - tail - (n - tail) % 256
    p, gr = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    p[lo:] = torch.randn(n - lo, generator=g, device="cuda")
    gr[lo:] = torch.randn(n - lo, generator=g, device="cuda").sign().bfloat16()
    state = [torch.zeros(n, dtype=torch.float32 if bits == 32 else torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.ones(-(-n // 256), device="cuda") for _ in range(2)] if bits == 8 else [None, None]
    cut = lambda t, k=lo: None if t is None else t[k:].clone()  # noqa: E731
    small = [cut(p), cut(gr), *[cut(t) for t in state], *[cut(t, lo // 256) for t in scale]]
    wrap = lambda t: None if t is None else [t]  # noqa: E731
    b.AdamW([p], [gr], *[[t] for t in state], *[wrap(t) for t in scale], seed=1).step(1e-2, beta1=0.5, beta2=0.5, step=1)
    b.AdamW([small[0]], [small[1]], [small[2]], [small[3]], wrap(small[4]), wrap(small[5]), seed=1).step(1e-2, beta1=0.5, beta2=0.5, step=1)
    assert torch.equal(p[lo:], small[0])
    for t, u in zip(state, small[2:4]):
        assert torch.equal(t[lo:], u)
    for t, u in zip(scale, small[4:]):
        assert t is None or torch.equal(t[lo // 256:], u)


def test_refusals():
    import ctypes
    b = sb()
    t = (b.sb_adamw_tensor * 1)()
    a = ctypes.c_void_p(0x1000)
    for k in ("param", "grad", "m", "v", "m_scale", "v_scale"):
        setattr(t[0], k, a)
    t[0].n = 4
    cfg, h = b.sb_adamw_config(0, 32, 0), b.sb_adamw_hyper(1e-3, 0.9, 0.999, 1e-8, 0.0, None, None)
    call = lambda n=1, c=cfg, hh=h, step=1, lst=t: b.sb_adamw_tensors(lst, n, ctypes.byref(c), ctypes.byref(hh), step, None)  # noqa: E731
    assert call(n=-1) == 1 and call(step=0) == 1 and b.sb_adamw_tensors(None, 1, ctypes.byref(cfg), ctypes.byref(h), 1, None) == 1
    assert call(c=b.sb_adamw_config(0, 16, 0)) == 1 and call(c=b.sb_adamw_config(0, 32, 2)) == 1
    for bad in ((float("nan"), 0.9, 0.999, 1e-8, 0.0), (1e-3, 1.0, 0.999, 1e-8, 0.0), (1e-3, 0.9, -0.1, 1e-8, 0.0), (1e-3, 0.9, 0.9, -1.0, 0.0), (1e-3, 0.9, 0.9, 1e-8, float("inf"))):
        assert call(hh=b.sb_adamw_hyper(*bad, None, None)) == 1
    assert "finite" in b.sb_last_error()
    for field, value, bits in (("param", 0x1002, 32), ("param", None, 32), ("grad", None, 32), ("m", 0x1001, 32), ("v", None, 8), ("m_scale", None, 8), ("shadow", 0x1001, 32)):
        bad = (b.sb_adamw_tensor * 1)(t[0])
        setattr(bad[0], field, value)
        assert call(c=b.sb_adamw_config(0, bits, 0), lst=bad) == 1, field
    t[0].n = -1
    assert call() == 2
    outs = (ctypes.c_void_p * 1)(a)
    t[0].n = 4
    assert b.sb_adamw_moments(t, 1, ctypes.byref(cfg), outs, outs, None) == 1
    assert b.sb_adamw_moments(t, 1, ctypes.byref(b.sb_adamw_config(0, 8, 0)), outs, None, None) == 1
    # an empty list, and one of empty tensors, is a step of nothing
    assert call(n=0) == 0
    t[0].n = 0
    assert call() == 0


def test_binding_refusals():
    import torch
    b = sb()
    p = torch.zeros(8)
    with pytest.raises(b.SBError):
        b.AdamW([], [], [], [])
    with pytest.raises(b.SBError):
        b.AdamW([p], [p], [p], [p, p])
    with pytest.raises(b.SBError):
        b.AdamW([p.half()], [p], [p], [p])
    with pytest.raises(b.SBError):
        b.AdamW([p], [torch.zeros(4)], [p], [p])
    with pytest.raises(b.SBError):
        b.AdamW([p], [p.double()], [p], [p])
    with pytest.raises(b.SBError):
        b.AdamW([torch.zeros(16)[::2]], [p], [p], [p])
    with pytest.raises(b.SBError):
        b.AdamW([p], [p], [p.to(torch.uint8)], [p.to(torch.uint8)], [torch.zeros(2)], [torch.zeros(1)])
    with pytest.raises(b.SBError):
        b.AdamW([p], [p], [p], [p]).step(1e-3)          # not on a CUDA device


def test_binding_holds_what_it_has_addresses_of():
    """The lists are the caller's to change: the tensors live on, and a call with unfit gradients leaves those of the call before."""
    import gc
    import weakref
    import torch
    b = sb()
    lists = [[torch.zeros(8) for _ in range(2)] for _ in range(5)]          # p, g, m, v, shadows
    lists[4] = [t.bfloat16() for t in lists[4]]
    a = b.AdamW(*lists[:4], shadows=lists[4])
    alive = [weakref.ref(t) for x in lists for t in x]
    before = [e.grad for e in a._list]
    for bad in ([torch.zeros(8)], [torch.zeros(8)] * 3, [torch.zeros(8), torch.zeros(4)], [torch.zeros(8), torch.zeros(8).bfloat16()], []):
        with pytest.raises(b.SBError):
            a.set_grads(bad)
        assert [e.grad for e in a._list] == before and a.cfg.grad_dtype == b.SB_DT_F32
    for x in lists:
        x.clear()
    gc.collect()
    assert all(w() is not None for w in alive)
    new = [torch.zeros(8).bfloat16() for _ in range(2)]
    a.set_grads(iter(new))
    assert [e.grad for e in a._list] == [t.data_ptr() for t in new] and a.cfg.grad_dtype == b.SB_DT_BF16


def test_binding_refuses_a_parameter_twice_and_scales_of_one_moment():
    import torch
    b = sb()
    p, q, c = torch.zeros(8), torch.zeros(8), torch.zeros(8, dtype=torch.uint8)
    with pytest.raises(b.SBError):
        b.AdamW([p, p], [q, q], [q, q], [q, q])
    for scales in (([torch.zeros(1)], None), (None, [torch.zeros(1)])):
        with pytest.raises(b.SBError):
            b.AdamW([p], [q], [c], [c], *scales)
    b.AdamW([torch.zeros(0), torch.zeros(0), p], [torch.zeros(0), torch.zeros(0), q], [torch.zeros(0), torch.zeros(0), q], [torch.zeros(0), torch.zeros(0), q])
