"""Residual gated feed-forward blocks inside a network, and its AdamW update: layer by layer and end to end against the formulas in 64 bits, the
different ways of running a step against one another, refusals and the partitioning table on the CPU."""
import ctypes

import numpy as np
import pytest

import sb_inputs as si

GATED = 10


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


def net(width=64, hidden=(96, 40), classes=10):
    return [(si.CONV3X3_RELU, 8), (si.MAXPOOL2, 0), (si.FC_RELU, width), *[(GATED, f) for f in hidden], (si.FC_RELU, 32), (si.FC, classes), (si.SOFTMAX_XENT, classes)]


def workload(layers, b=4, R=2, K=2, H=8, W=8, C=8):
    return si.Workload("gated", layers, H, W, C, b, R, K)


def make_params(wl, seed=0):
    """He-normal weights; the blocks' vectors around one (the gate around a half)"""
    rng = np.random.default_rng(seed)
    out, c, feat = [], wl.C, wl.H * wl.W * wl.C
    h, w = wl.H, wl.W
    for kind, o in wl.layers:
        n = lambda *s, std=1.0: (rng.standard_normal(s) * std).astype(np.float32)  # noqa: E731
        if kind == si.CONV3X3_RELU:
            out.append({"w": n(o, 3, 3, c, std=(2 / (9 * c)) ** 0.5), "b": n(o, std=0.05)})
            c = o
            feat = h * w * c
        elif kind == si.MAXPOOL2:
            h, w = h // 2, w // 2
            feat = h * w * c
            out.append(None)
        elif kind in (si.FC_RELU, si.FC):
            out.append({"w": n(o, feat, std=(2 / feat) ** 0.5), "b": n(o, std=0.05)})
            feat = o
        elif kind == GATED:
            out.append({"gate_up": n(2 * o, feat, std=feat ** -0.5), "down": n(feat, o, std=o ** -0.5), "w_pre": 1 + n(feat, std=0.1),
                        "w_post": 1 + n(feat, std=0.1), "gate": 0.5 + n(feat, std=0.1), "scale": 1 + n(feat, std=0.1)})
        else:
            out.append(None)
    return out


def rms(v):
    return v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()


def block(x, p):
    import torch
    g, u = (rms(x) * p["w_pre"] @ p["gate_up"].t()).chunk(2, 1)
    return p["scale"] * x + p["gate"] * (p["w_post"] * rms((torch.nn.functional.silu(g) * u) @ p["down"].t()))


def reference(wl, params, x, labels):
    """loss and the gradients of every parameter, in 64 bits"""
    import torch
    F = torch.nn.functional
    ps = [None if p is None else {k: torch.from_numpy(np.asarray(v)).double().requires_grad_() for k, v in p.items()} for p in params]
    a = torch.from_numpy(x).double().permute(0, 3, 1, 2)
    for (kind, _), p in zip(wl.layers, ps):
        if kind == si.CONV3X3_RELU:
            a = F.relu(F.conv2d(a, p["w"].permute(0, 3, 1, 2), p["b"], padding=1))
        elif kind == si.MAXPOOL2:
            a = F.max_pool2d(a, 2)
        else:
            if a.dim() == 4:
                a = a.permute(0, 2, 3, 1).reshape(a.shape[0], -1)
            if kind in (si.FC_RELU, si.FC):
                a = a @ p["w"].t() + p["b"]
                a = F.relu(a) if kind == si.FC_RELU else a
            elif kind == GATED:
                a = block(a, p)
    loss = F.cross_entropy(a, torch.from_numpy(labels).long())
    loss.backward()
    return loss.item(), [None if p is None else {k: v.grad.numpy() for k, v in p.items()} for p in ps]


def batch(wl, seed=1):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((wl.B, wl.H, wl.W, wl.C)).astype(np.float32), rng.integers(0, wl.layers[-1][1], wl.B).astype(np.int32)


def model(b, wl, params, precision, flags=0):
    m = b.Model.from_workload(wl, precision=precision, flags=flags)
    m.load_params(params, si.shard_bounds)
    return m


def device(wl, x, y, bf16):
    import torch
    t = torch.from_numpy(x).cuda()
    t = t.to(torch.bfloat16) if bf16 else t
    return list(t.split(wl.b)), list(torch.from_numpy(y).cuda().split(wl.b))


def frob(a, r):
    return float(np.linalg.norm(np.asarray(a, np.float64) - r) / (np.linalg.norm(r) + 1e-30))


@pytest.mark.gpu
@pytest.mark.parametrize("width,hidden,b", [(64, (96, 40), 4), (33, (17,), 3), (520, (1368, 64), 40)])
def test_gradients_of_a_network_in_float(width, hidden, b):
    lib = sb()
    wl = workload(net(width, hidden), b=b)
    params = make_params(wl)
    x, y = batch(wl)
    loss, grads = reference(wl, params, x, y)
    m = model(lib, wl, params, lib.SB_FP32)
    m.debug_poison()
    m.forward(*device(wl, x, y, False))
    m.backward()
    # float sums of some thousand products and the network's depth: the bound of the float mode's other networks
    assert abs(m.loss() - loss) <= 1e-5 * max(1, abs(loss))
    for li, (got, ref) in enumerate(zip(m.gather_params(lib.SB_T_GRAD_W, lib.SB_T_GRAD_B), grads)):
        for k in ref or {}:
            assert np.max(np.abs(got[k].reshape(ref[k].shape) - ref[k])) <= 1e-4 * np.max(np.abs(ref[k])), (li, k)
    assert m.debug_check_guards()[0] == 0
    m.close()


@pytest.mark.gpu
@pytest.mark.parametrize("below", ["fc", "pool", "conv", "block"])
@pytest.mark.parametrize("bf16", [False, True])
def test_one_layer(below, bf16):
    """The block alone, on given activations and gradient: its output, the gradient it hands down (with the mask of a ReLU layer below), its parameters'
    gradients.  In bf16 each of w_pre N(x), GU, H, the block's output, y -- and back df, dG and dU, dn, dx twice -- is rounded once, by half a step, 2^-8 of
    the value; a norm behind a rounding at most doubles it relative to the row, and roundings add up: eight halves of a step for y, sixteen for gradients."""
    import torch
    lib = sb()
    head = {"fc": [(si.FC_RELU, 96)], "pool": [(si.CONV3X3_RELU, 8), (si.MAXPOOL2, 0)], "conv": [(si.CONV3X3_RELU, 8)], "block": [(si.FC_RELU, 96), (GATED, 64)]}[below]
    wl = workload(head + [(GATED, 104), (si.FC, 10), (si.SOFTMAX_XENT, 10)], b=9, H=4, W=6)
    at = len(head)
    params = make_params(wl, 3)
    m = model(lib, wl, params, lib.SB_BF16 if bf16 else lib.SB_FP32)
    D = params[at]["w_pre"].size
    g = torch.Generator().manual_seed(5)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn(wl.B, D, generator=g)
    x = (x.relu() if below in ("fc", "conv") else x).to(dt)
    dy = torch.randn(wl.B, D, generator=g).to(dt)
    x_np, dy_np = x.float().numpy(), dy.float().numpy()
    if below in ("pool", "conv"):
        for r in range(wl.R):
            m.write(lib.SB_T_ACT, at - 1, r, x_np[r * wl.b:(r + 1) * wl.b])
    else:
        m.write(lib.SB_T_ACT, at - 1, 0, x_np)
    m.forward_layers(at, at)
    m.write(lib.SB_T_DACT, at, 0, dy_np)
    m.backward_layers(at, at)
    torch.cuda.synchronize()
    rnd = (lambda v: torch.from_numpy(v).to(torch.bfloat16).double()) if bf16 else (lambda v: torch.from_numpy(v).double())
    p = {k: (rnd(v) if k in ("gate_up", "down") else torch.from_numpy(v).double()).requires_grad_() for k, v in params[at].items()}
    xr = x.double().requires_grad_()
    y = block(xr, p)
    y.backward(dy.double())
    dx = xr.grad * (x > 0) if below in ("fc", "conv") else xr.grad
    u = 2.0 ** -8 if bf16 else 1e-6
    assert frob(m.read(lib.SB_T_ACT, at, 0), y.detach().numpy()) <= 8 * u
    got = [m.read(lib.SB_T_DACT, at - 1, r) for r in range(wl.R)] if below in ("pool", "conv") else [m.read(lib.SB_T_DACT, at - 1, 0)]
    assert frob(np.concatenate([a.reshape(-1) for a in got]), dx.reshape(-1).numpy()) <= 16 * u
    grads = m.gather_params(lib.SB_T_GRAD_W, lib.SB_T_GRAD_B)[at]
    for k in p:
        assert frob(grads[k], p[k].grad.numpy()) <= 16 * u, k
    m.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
def test_ways_of_running_a_step_agree(bf16):
    """Separate calls, the replayed iteration and the call from host buffers leave the same parameters and momenta, bit for bit."""
    import torch
    lib = sb()
    wl = workload(net(), b=8)
    params = make_params(wl)
    batches = [batch(wl, s) for s in range(4)]
    results = []
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for way in ("calls", "graph", "host"):
            m = model(lib, wl, params, lib.SB_BF16 if bf16 else lib.SB_FP32)
            xs, ys = device(wl, *batches[0], bf16)
            losses = []
            for x, y in batches:
                if way == "host":
                    t = torch.from_numpy(x).to(torch.bfloat16 if bf16 else torch.float32).pin_memory()
                    losses.append(m.train_step_host(t, torch.from_numpy(y).pin_memory(), 0.01, 0.9))
                    continue
                for dst, src in zip((*xs, *ys), (*device(wl, x, y, bf16)[0], *device(wl, x, y, bf16)[1])):
                    dst.copy_(src)
                if way == "graph":
                    m.graph_step(xs, ys, 0.01, 0.9)
                else:
                    m.forward(xs, ys)
                    m.backward()
                    m.sgd_step(0.01, 0.9)
                losses.append(m.loss())
            results.append((losses, m.gather_params(lib.SB_T_WEIGHT, lib.SB_T_BIAS), m.gather_params(lib.SB_T_MOM_W, lib.SB_T_MOM_B)))
            assert m.debug_check_guards()[0] == 0
            m.close()
    for other in results[1:]:
        assert other[0] == results[0][0]
        for a, c in zip(results[0][1] + results[0][2], other[1] + other[2]):
            for k in a or {}:
                assert np.array_equal(a[k], c[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
def test_adamw_steps_of_a_model(bf16):
    """forward, backward, adamw_step on a network with blocks: every parameter and moment from the model's own gradients, by the formulas."""
    lib = sb()
    wl = workload(net(), b=8)
    m = model(lib, wl, make_params(wl), lib.SB_BF16 if bf16 else lib.SB_FP32, lib.SB_FLAG_ADAMW)
    h = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
    U = 2.0 ** -24
    zero = lambda ps: [None if p is None else {k: np.zeros_like(v, dtype=np.float64) for k, v in p.items()} for p in ps]  # noqa: E731
    ps = m.gather_params(lib.SB_T_WEIGHT, lib.SB_T_BIAS)
    ms, vs = zero(ps), zero(ps)
    for t in (1, 2, 3):
        m.forward(*device(wl, *batch(wl, t), bf16))
        m.backward()
        gs = m.gather_params(lib.SB_T_GRAD_W, lib.SB_T_GRAD_B)
        m.adamw_step(step=t, **h)
        new = [m.gather_params(a, c) for a, c in ((lib.SB_T_WEIGHT, lib.SB_T_BIAS), (lib.SB_T_MOM_W, lib.SB_T_MOM_B), (lib.SB_T_VAR_W, lib.SB_T_VAR_B))]
        for li, g in enumerate(gs):
            for k in g or {}:
                gd = g[k].astype(np.float64)
                m_ref, v_ref = 0.9 * ms[li][k] + 0.1 * gd, 0.99 * vs[li][k] + 0.01 * gd * gd
                step = h["lr"] / (1 - 0.9 ** t) * m_ref / (np.sqrt(v_ref / (1 - 0.99 ** t)) + h["eps"])
                p_ref = (1 - h["lr"] * h["weight_decay"]) * ps[li][k].astype(np.float64) - step
                m_err = 3 * U * (0.9 * np.abs(ms[li][k]) + 0.1 * np.abs(gd))
                assert np.all(np.abs(new[1][li][k] - m_ref) <= m_err + 1e-45)
                assert np.all(np.abs(new[2][li][k] - v_ref) <= 5 * U * v_ref + 1e-45)
                slope = h["lr"] / (1 - 0.9 ** t) / (np.sqrt(v_ref / (1 - 0.99 ** t)) + h["eps"])
                assert np.all(np.abs(new[0][li][k] - p_ref) <= 4 * U * (np.abs(p_ref) + np.abs(step)) + slope * m_err + 16 * U * np.abs(step) + 1e-45), (li, k)
        ps, ms, vs = new[0], *[[None if p is None else {k: v.astype(np.float64) for k, v in p.items()} for p in side] for side in new[1:]]
    if bf16:
        for part in (0, 1):
            w = m.read(lib.SB_T_WEIGHT, 3, part)
            assert np.array_equal(m.read(lib.SB_T_SHADOW_W, 3, part), lib.bf16_bits_to_f32(lib.f32_to_bf16_bits(w)).reshape(w.shape))
    xs, ys = device(wl, *batch(wl, 9), bf16)
    for call in (lambda: m.sgd_step(0.1, 0.9), lambda: m.graph_step(xs, ys, 0.1, 0.9), lambda: m.train_step_host(*batch(wl, 9), 0.1, 0.9)):
        with pytest.raises(lib.SBError) as e:
            call()
        assert e.value.status == 6
    with pytest.raises(lib.SBError):
        m.adamw_step(1e-3, step=0)
    m.close()
    m = model(lib, wl, make_params(wl), lib.SB_FP32)
    with pytest.raises(lib.SBError) as e:
        m.adamw_step(1e-3)
    assert e.value.status == 6
    with pytest.raises(lib.SBError):
        m.read(lib.SB_T_VAR_W, 3, 0)
    m.close()


@pytest.mark.gpu
def test_operators_together():
    """A block and its training as a program without a model runs them: both norms, the feed-forward block, their gradients, one AdamW step over
    all its tensors; against the formulas in 64 bits.  Tolerances as in the operators' own float tests, added up over the chain."""
    import torch
    lib = sb()
    rows, d, f = 70, 136, 200
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).cuda()  # noqa: E731
    p = {"w_pre": 1 + rnd(d, std=0.1), "w_post": 1 + rnd(d, std=0.1), "gate": 0.5 + rnd(1, d, std=0.1), "scale": 1 + rnd(d, std=0.1),
         "gate_up": rnd(2 * f, d, std=d ** -0.5), "down": rnd(d, f, std=f ** -0.5)}
    x, dy = rnd(rows, d), rnd(rows, d)
    _, n, st1 = lib.norm_forward(x, p["w_pre"], save=True)
    out, gu = lib.ffn_forward(n, p["gate_up"], p["down"], save=True)
    y, _, st2 = lib.norm_forward(x, None, out, p["w_post"], p["gate"], p["scale"], save=True)
    b2 = lib.norm_backward(dy, None, st2, x, None, out, p["w_post"], p["gate"], p["scale"])
    dn, dgu, dd = lib.ffn_backward(b2["df"], n, gu, p["gate_up"], p["down"])
    b1 = lib.norm_backward(b2["dx"], dn, st1, x, p["w_pre"])
    grads = {"w_pre": b1["dw_pre"], "w_post": b2["dw_post"], "gate": b2["dgate"], "scale": b2["dscale"], "gate_up": dgu, "down": dd}
    xd = x.double().requires_grad_()
    pd = {k: v.double().requires_grad_() for k, v in p.items()}
    ref = block(xd, pd)
    ref.backward(dy.double())
    close = lambda a, r, tol: float((a.double() - r).norm() / r.norm()) <= tol  # noqa: E731
    assert close(y, ref.detach(), 1e-5) and close(b1["dx"], xd.grad, 1e-5)
    for k in p:
        assert close(grads[k], pd[k].grad, 1e-5), k
    before = {k: v.double().clone() for k, v in p.items()}
    names = list(p)
    opt = lib.AdamW([p[k] for k in names], [grads[k] for k in names], [torch.zeros_like(p[k]) for k in names], [torch.zeros_like(p[k]) for k in names])
    opt.step(1e-3, step=1)
    for k in names:
        gr = grads[k].double()
        want = before[k] * (1 - 1e-3 * 0.01) - 1e-3 * gr / (gr.abs() + 1e-8)
        assert float((p[k].double() - want).abs().max()) <= 1e-6
    lib.ops_check()


def test_partitioning_table_and_exchange():
    """A block stays whole: a shard node in front of it gathers a split layer's columns; its parameters are reduced like those of a layer kept whole."""
    lib = sb()
    layers = net()
    nodes = lib.partition(layers, 8, 8, 8, 2)
    at = [k for k, n in enumerate(nodes) if n["node"] == lib.SB_NODE_LAYER and layers[n["layer"]][0] == GATED]
    assert [(nodes[k]["shards"], nodes[k]["dim"], nodes[k]["dimF"]) for k in at] == [(1, 64, 64)] * 2
    assert nodes[at[0] - 1]["node"] == lib.SB_NODE_SHARD and nodes[at[1] - 1]["node"] == lib.SB_NODE_LAYER
    msgs = lib.exchange_plan(layers, 8, 8, 8, 4, 4, 2)
    assert {m["src"] for m in msgs if m["layer"] == 3 and m["kind"] == lib.SB_X_ALLREDUCE_GROUPS} == {-1}
    assert not [m for m in msgs if m["layer"] == 3 and m["kind"] == lib.SB_X_ALLREDUCE]
    alone = lib.exchange_plan(layers, 8, 8, 8, 4, 3, 1)
    assert [m for m in alone if m["layer"] == 3] and all(m["kind"] == lib.SB_X_ALLREDUCE for m in alone if m["layer"] == 3)


def test_validation():
    lib = sb()

    def status(layers, H=8, W=8, C=8, flags=0, K=2):
        arr = lib._layers_array(layers)
        c = lib.sb_config(H, W, C, 4, 2, K, 1, flags)
        n = ctypes.c_size_t()
        return lib.sb_model_bytes(arr, len(layers), ctypes.byref(c), ctypes.byref(n)), n.value

    good, size = status(net())
    assert good == 0
    assert status(net(), flags=lib.SB_FLAG_ADAMW)[1] > size
    assert status(net()[2:])[0] == 0                                                              # behind a first FC layer
    assert status([(GATED, 8), (si.FC, 4), (si.SOFTMAX_XENT, 4)])[0] == 3                          # the first layer
    assert status([(si.FC_RELU, 8), (GATED, 0), (si.FC, 4), (si.SOFTMAX_XENT, 4)])[0] == 2          # no hidden width
    assert status([(si.FC_RELU, 8), (si.FC, 4), (GATED, 4), (si.SOFTMAX_XENT, 4)])[0] in (2, 3)     # behind the logits
    assert status(net(), flags=lib.SB_FLAG_MODULO_SCHEDULE)[0] == 3
    assert status([(si.CONV3X3_RELU, 64), (GATED, 8), (si.FC, 4), (si.SOFTMAX_XENT, 4)], H=32, W=32)[0] == 3      # 65536 columns
    assert status([(si.FC_RELU, 8), (GATED, 8), (si.DROPOUT, 100), (si.FC, 4), (si.SOFTMAX_XENT, 4)])[0] == 3       # dropout follows an FC layer
    assert lib.sb_adamw_step(None, None, 1, None) == 1
