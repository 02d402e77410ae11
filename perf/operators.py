"""The operators of a residual gated feed-forward block and of its training, each through the calls a user's program makes.

    op "ffn"      gated feed-forward block: forward (with or without what the backward pass needs) or backward
    op "norm"     norms before and after a block, fused with the block's gate and the residual scale: forward or backward
    op "adamw"    one AdamW step over a list of tensors, states in 32 or 8 bits

With R rows, width D and hidden width F:

    ffn     GU = X Wgu^T, G and U its halves, H = a(G) * U, Y = H Wd^T
    norm    y = s * x + g * (wpost * N(f)),  n = wpre * N(y)
    adamw   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
            p <- (1 - lr wd) p - lr m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps)
"""
from __future__ import annotations

import math

import torch

own = False

ACTS = ("silu", "gelu", "relu")
BETA1, BETA2, EPS, DECAY, LR = 0.9, 0.999, 1e-8, 0.1, 1e-3
NORM_EPS = 1e-6
BLOCK = 256            # elements of a tensor that share one scale of the 8-bit states
M32 = 0xFFFFFFFF

# tensors of the networks that this repository trains: weights and biases, layer by layer (input channels, output channels)
_VGG_CONV = [(3, 64), (64, 64), (64, 128), (128, 128), (128, 256), (256, 256), (256, 256), (256, 512), (512, 512), (512, 512), (512, 512),
             (512, 512), (512, 512)]


def _net(name):
    conv, fc = {
        "tiny": ([(3, 16), (16, 32)], [(2048, 64), (64, 10)]),
        "paper": ([(3, 64), (64, 64), (64, 128), (128, 128), (128, 256), (256, 256), (256, 256)], [(4096, 1024), (1024, 1024), (1024, 10)]),
        "vgg16_32": (_VGG_CONV, [(512, 4096), (4096, 4096), (4096, 10)]),
        "vgg16_224": (_VGG_CONV, [(25088, 4096), (4096, 4096), (4096, 1000)]),
    }[name]
    return [n for i, o in conv for n in (9 * i * o, o)] + [n for i, o in fc for n in (i * o, o)]


def _sizes(case):
    if case["net"] != "list":
        return _net(case["net"])
    # a list of `tensors` ragged tensors between 1 and about `largest` elements
    k = case["tensors"]
    return [max(1, int(case["largest"] ** ((i * 7 % k + 1) / k)) - i % 3) for i in range(k)]


def _ffn(name, way, dtype, rows, d, f, act):
    return dict(name=name, op="ffn", way=way, dtype=dtype, rows=rows, d=d, f=f, act=act)


def _norm(name, way, dtype, kind, rows, d, groups, pre=True, post=True, scale=True):
    return dict(name=name, op="norm", way=way, dtype=dtype, kind=kind, rows=rows, d=d, groups=groups, pre=pre, post=post, scale=scale)


def _adamw(name, net, bits, grad, shadow, tensors=0, largest=0):
    return dict(name=name, op="adamw", net=net, bits=bits, grad=grad, shadow=shadow, tensors=tensors, largest=largest)


def listed():
    return [
        # one example answered: the block is as long as its weights take to read
        _ffn("ffn_answer_r1_bf16", "answer", "bf16", 1, 4096, 8192, "silu"),
        # a ragged batch of the small head, forward of a training step
        _ffn("ffn_forward_r111_bf16", "forward", "bf16", 111, 512, 1368, "gelu"),
        # a large batch, forward of a training step
        _ffn("ffn_forward_r8192_bf16", "forward", "bf16", 8192, 4096, 8192, "silu"),
        # its backward pass, a batch that fills no tile
        _ffn("ffn_backward_r4000_bf16", "backward", "bf16", 4000, 4096, 8192, "silu"),
        # float mode, widths without any alignment, backward
        _ffn("ffn_backward_r250_fp32", "backward", "fp32", 250, 1023, 2731, "gelu"),
        # the norm in front of the first block while answering eight examples
        _norm("norm_pre_r8_bf16", "forward", "bf16", "rms", 8, 4096, 0, post=False, scale=False),
        # between two blocks of a training step: both norms, a gate per image (16 positions each), the residual scale
        _norm("norm_both_r16384_bf16", "forward", "bf16", "rms", 16384, 4096, 1024),
        # its backward pass
        _norm("norm_both_backward_r16384_bf16", "backward", "bf16", "rms", 16384, 4096, 1024),
        # layer norms in float at an odd width, one gate for all rows, backward
        _norm("norm_both_backward_r999_fp32", "backward", "fp32", "layer", 999, 1001, 1),
        # the smallest network's eight tensors
        _adamw("adamw_tiny_32", "tiny", 32, "fp32", True),
        # the large network, states in 32 bits, as the float gradients come
        _adamw("adamw_vgg16_224_32", "vgg16_224", 32, "fp32", True),
        # the same with states in 8 bits and bf16 gradients
        _adamw("adamw_vgg16_224_8", "vgg16_224", 8, "bf16", True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["ffn", "ffn", "ffn", "norm", "norm", "adamw"])
    if op == "ffn":
        way, act = rng.choice(["answer", "forward", "backward"]), rng.choice(ACTS)
        kind = rng.choice(["bf16", "bf16", "bf16", "odd", "fp32"])
        if kind == "bf16":
            rows = _log_int(rng, 1, 64) if way == "answer" else _log_int(rng, 16, 8192)
            d, f = 8 * _log_int(rng, 16, 512), 8 * _log_int(rng, 16, 1024)
            if way == "backward":
                rows = min(rows, 4000)
        else:
            rows, d, f = _log_int(rng, 1, 512), _log_int(rng, 40, 1100), _log_int(rng, 40, 2800)
        return _drawn(_ffn, way, "fp32" if kind == "fp32" else "bf16", rows, d, f, act)
    if op == "norm":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        pre, post = rng.choice([(True, True), (True, True), (True, False), (False, True)])
        rows, d = _log_int(rng, 1, 16384), _log_int(rng, 32, 4096)
        if rng.random() < 0.7:
            d = max(32, d // 8 * 8)
        rows = max(1, min(rows, (16384 * 4096 if dtype == "bf16" else 8192 * 4096) // d))
        groups = rng.choice([g for g in (0, 1, rows, rows // 2, rows // 16) if g == 0 or (g > 0 and rows % g == 0)]) if post else 0
        return _drawn(_norm, rng.choice(["forward", "backward"]), dtype, rng.choice(["rms", "layer"]), rows, d, groups, pre, post,
                      post and rng.random() < 0.6)
    net = rng.choice(["paper", "vgg16_32", "list", "list", "list"])
    return _drawn(_adamw, net, rng.choice([32, 8]), rng.choice(["fp32", "bf16"]), rng.random() < 0.6,
                  *((_log_int(rng, 1, 400), _log_int(rng, 100, 1 << 20)) if net == "list" else (0, 0)))


def _drawn(make, *a):
    c = make("", *a)
    del c["name"]
    return c


def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        # parameter in and out, gradient in, both moments in and out, the bf16 copy out
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (8 + (4 if case["grad"] == "fp32" else 2) + state + (2 if case["shadow"] else 0)), "flops": 14 * n}
    e, R, D = 2 if case["dtype"] == "bf16" else 4, case["rows"], case["d"]
    if case["op"] == "ffn":
        F = case["f"]
        if case["way"] == "backward":
            # x, dy, GU, both weights in; dx and both weight gradients out
            return {"bytes": e * (3 * R * D + 2 * R * F + 6 * D * F), "flops": 12 * R * D * F}
        return {"bytes": e * (2 * R * D + 3 * D * F + (2 * R * F if case["way"] == "forward" else 0)), "flops": 6 * R * D * F}
    both, vectors = case["post"], D * (case["pre"] + case["post"] + case["scale"] + case["groups"])
    if case["way"] == "forward":
        # x (and f) in; y (where it is not x) and n out
        return {"bytes": e * R * D * (1 + 2 * both + case["pre"]) + 4 * vectors, "flops": 12 * R * D}
    # x (and f), the gradients of y and n in; those of x (and f) out
    return {"bytes": e * R * D * (3 + 2 * both + case["pre"]) + 8 * vectors, "flops": 30 * R * D}


# ---- inputs --------------------------------------------------------------------------------------------------------


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape, std=1.0: torch.randn(*shape, generator=g, device="cuda") * std  # noqa: E731
    if case["op"] == "adamw":
        _prepare_adamw(s, case, seed, normal, g)
        return s
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    R, D = case["rows"], case["d"]
    s.x = normal(R, D).to(dt)
    if case["op"] == "ffn":
        F = case["f"]
        s.w_gate_up = normal(2 * F, D, std=1.0 / math.sqrt(D)).to(dt)
        s.w_down = normal(D, F, std=1.0 / math.sqrt(F)).to(dt)
        if case["way"] == "backward":
            # what the forward pass has kept, and the gradient of a mean over the rows
            s.gu = (s.x.float() @ s.w_gate_up.float().t()).to(dt)
            s.dy = normal(R, D, std=1.0 / R).to(dt)
        return s
    s.f = normal(R, D, std=0.5).to(dt) if case["post"] else None
    s.w_pre = 1.0 + normal(D, std=0.1) if case["pre"] else None
    s.w_post = 1.0 + normal(D, std=0.1) if case["post"] else None
    s.gate = 0.5 + normal(case["groups"], D, std=0.2) if case["groups"] else None
    s.scale = 1.0 + normal(D, std=0.05) if case["scale"] else None
    if case["way"] == "backward":
        s.dy = normal(R, D).to(dt)
        s.dn = normal(R, D).to(dt) if case["pre"] else None
        # what the forward pass has kept: mean and 1 / deviation of every row of f and of y
        s.stats = _norm_stats(s, case)
    return s


def _norm_stats(s, case):
    st = torch.zeros(case["rows"], 4, device="cuda", dtype=torch.float64)
    x = s.x.double()
    if case["post"]:
        mean, inv, hat = _normed(s.f.double(), case["kind"])
        st[:, 0], st[:, 1] = mean[:, 0], inv[:, 0]
        x = _residual(x, hat * s.w_post.double(), s.gate, s.scale, case)
    if case["pre"]:
        mean, inv, _ = _normed(x, case["kind"])
        st[:, 2], st[:, 3] = mean[:, 0], inv[:, 0]
    return st.float()


def _prepare_adamw(s, case, seed, normal, g):
    s.sizes, s.step, s.seed = _sizes(case), 100, seed
    gdt = torch.bfloat16 if case["grad"] == "bf16" else torch.float32
    s.p = [normal(n, std=0.05) for n in s.sizes]
    s.shadow = [p.to(torch.bfloat16) for p in s.p] if case["shadow"] else None
    # gradients of very different sizes within a tensor, as layers see them; moments of a run under way
    s.g = [(normal(n, std=1e-3) * torch.exp(normal(n))).to(gdt) for n in s.sizes]
    m = [normal(n, std=3e-4) * torch.exp(normal(n)) for n in s.sizes]
    v = [torch.exp(2.0 * normal(n)) * 1e-6 for n in s.sizes]
    if case["bits"] == 32:
        s.m, s.v, s.m_scale, s.v_scale = m, v, None, None
    else:
        s.m, s.m_scale = map(list, zip(*map(_encode_m, m)))
        s.v, s.v_scale = map(list, zip(*(_encode_v(b, _half_words(n, seed, i, 0, b.device)) for i, (n, b) in enumerate(zip(s.sizes, v)))))
    s.optimizer = _optimizer(s) if own else None


def _optimizer(s):
    from paper_2112_15317_b200 import binding as sb

    return sb.AdamW(s.p, s.g, s.m, s.v, s.m_scale, s.v_scale, shadows=s.shadow, seed=s.seed)


# ---- a pass --------------------------------------------------------------------------------------------------------


def run(s):
    case = s.case
    if own:
        return _run_own(s, case)
    if case["op"] == "ffn":
        return _ffn_plain(s, case, torch.float32)
    if case["op"] == "norm":
        return _norm_plain(s, case, torch.float32)
    return _adamw_plain(s, case)


def _run_own(s, case):
    from paper_2112_15317_b200 import binding as sb

    if case["op"] == "ffn":
        act = {"silu": sb.SB_ACT_SILU, "gelu": sb.SB_ACT_GELU, "relu": sb.SB_ACT_RELU}[case["act"]]
        if case["way"] == "answer":
            return {"y": sb.ffn_forward(s.x, s.w_gate_up, s.w_down, act)}
        if case["way"] == "forward":
            y, gu = sb.ffn_forward(s.x, s.w_gate_up, s.w_down, act, save=True)
            return {"y": y, "gu": gu}
        dx, dw_gate_up, dw_down = sb.ffn_backward(s.dy, s.x, s.gu, s.w_gate_up, s.w_down, act)
        return {"dx": dx, "dw_gate_up": dw_gate_up, "dw_down": dw_down}
    if case["op"] == "norm":
        kind = sb.SB_NORM_RMS if case["kind"] == "rms" else sb.SB_NORM_LAYER
        if case["way"] == "forward":
            y, n = sb.norm_forward(s.x, s.w_pre, s.f, s.w_post, s.gate, s.scale, kind, NORM_EPS)
            return {"y": y if case["post"] else None, "n": n}
        return sb.norm_backward(s.dy, s.dn, s.stats, s.x, s.w_pre, s.f, s.w_post, s.gate, s.scale, kind)
    s.step += 1
    s.optimizer.step(LR, BETA1, BETA2, EPS, DECAY, s.step)
    m, v = (s.m, s.v) if case["bits"] == 32 else s.optimizer.moments()
    return _adamw_outputs(s, m, v)


def _adamw_outputs(s, m, v):
    # the large tensors one by one, the small ones in one list each
    pick = sorted(range(len(s.sizes)), key=lambda i: -s.sizes[i])[:12]
    out = {"p": [s.p[i] for i in pick], "m": [m[i] for i in pick], "v": [v[i] for i in pick]}
    if s.shadow is not None:
        out["shadow"] = [s.shadow[i] for i in pick]
    return out


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _act(g, name):
    """a(g) and its derivative"""
    if name == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _ffn_plain(s, case, t):
    dt, F = s.x.dtype, case["f"]
    x, wgu, wd = s.x.to(t), s.w_gate_up.to(t), s.w_down.to(t)
    if case["way"] != "backward":
        gu = x @ wgu.t()
        a, _ = _act(gu[:, :F], case["act"])
        y = ((a * gu[:, F:]) @ wd.t()).to(dt)
        return {"y": y} if case["way"] == "answer" else {"y": y, "gu": gu.to(dt)}
    dy, g, u = s.dy.to(t), s.gu[:, :F].to(t), s.gu[:, F:].to(t)
    a, da = _act(g, case["act"])
    dh = dy @ wd
    dgu = torch.cat([dh * u * da, dh * a], 1)
    return {"dx": (dgu @ wgu).to(dt), "dw_gate_up": (dgu.t() @ x).to(dt), "dw_down": (dy.t() @ (a * u)).to(dt)}


def _normed(v, kind):
    """mean (0 for rms), 1 / deviation and the normalised rows"""
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    c = v - mean
    inv = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + NORM_EPS)
    return mean, inv, c * inv


def _gated(v, gate, case):
    """v times the gate of its group of rows"""
    if gate is None:
        return v
    return (v.view(case["groups"], -1, case["d"]) * gate.to(v.dtype)[:, None, :]).view_as(v)


def _residual(x, p, gate, scale, case):
    return (x if scale is None else x * scale.to(x.dtype)) + _gated(p, gate, case)


def _norm_grad(dz, hat, inv, kind):
    """gradient of the normalised vector's input, dz being that of the normalised vector"""
    r = dz - hat * (dz * hat).mean(1, keepdim=True)
    if kind == "layer":
        r = r - dz.mean(1, keepdim=True)
    return r * inv


def _norm_plain(s, case, t):
    dt, kind, R = s.x.dtype, case["kind"], case["rows"]
    x = s.x.to(t)
    y = x
    if case["post"]:
        _, inv_f, hat_f = _normed(s.f.to(t), kind)
        p = hat_f * s.w_post.to(t)
        y = _residual(x, p, s.gate, s.scale, case)
    if case["pre"]:
        _, inv_y, hat_y = _normed(y, kind)
    if case["way"] == "forward":
        return {"y": y.to(dt) if case["post"] else None, "n": (hat_y * s.w_pre.to(t)).to(dt) if case["pre"] else None}
    out = dict(dx=None, df=None, dw_pre=None, dw_post=None, dgate=None, dscale=None)
    d = s.dy.to(t)
    if case["pre"]:
        dn = s.dn.to(t)
        out["dw_pre"] = (dn * hat_y).sum(0)
        d = d + _norm_grad(dn * s.w_pre.to(t), hat_y, inv_y, kind)
    out["dx"] = (d if s.scale is None else d * s.scale.to(t)).to(dt)
    if s.scale is not None:
        out["dscale"] = (d * x).sum(0)
    if case["post"]:
        if s.gate is not None:
            out["dgate"] = (d * p).view(case["groups"], R // case["groups"], case["d"]).sum(1)
        dp = _gated(d, s.gate, case)
        out["dw_post"] = (dp * hat_f).sum(0)
        out["df"] = _norm_grad(dp * s.w_post.to(t), hat_f, inv_f, kind).to(dt)
    return out if t == torch.float64 else {k: v if v is None or v.dtype == dt else v.float() for k, v in out.items()}


# 8-bit moments.  Each block of 256 elements has a scale, a power of two.  The first moment is held as e4m3 (four bits of
# exponent, three of mantissa and a sign), the second, never negative, with five bits of exponent and three of mantissa;
# that one is rounded up or down by chance (a step moves it by a thousandth, less than half a code), with 16 random bits
# for each element from the Philox-4x32-10 generator: words of counter (element / 8, tensor, step), key = seed.


def _blocks(a, fill=0.0):
    n = a.numel()
    out = torch.full((-(-n // BLOCK) * BLOCK,), fill, dtype=a.dtype, device=a.device)
    out[:n] = a
    return out.view(-1, BLOCK)


def _power(a):
    """per block: the power of two at or below the largest finite magnitude (2^-100 at least)"""
    top = torch.where(torch.isfinite(a), a.abs(), torch.zeros_like(a)).amax(1).clamp(min=2.0 ** -100).float()
    return (top.view(torch.int32) & 0x7F800000).view(torch.float32)


def _encode_m(a):
    b = _blocks(a)
    scale = _power(b) * 2.0 ** -7
    code = (b / scale[:, None]).to(torch.float8_e4m3fn)
    return code.reshape(-1)[: a.numel()].contiguous(), scale


def _decode_m(code, scale):
    return (_blocks(code.float()) * scale[:, None]).reshape(-1)[: code.numel()]


def _encode_v(a, half):
    b = _blocks(a)
    scale = _power(b)
    z = (b / scale[:, None]) * 2.0 ** -97
    code = (z.view(torch.int32).to(torch.int64) + (_blocks(half) << 4)) >> 20
    code = torch.where(torch.isfinite(b), code.clamp(max=254), torch.full_like(code, 255)).to(torch.uint8)
    return code.reshape(-1)[: a.numel()].contiguous(), scale


def _decode_v(code, scale):
    b = _blocks(code)
    v = (b.to(torch.int32) << 20).view(torch.float32) * 2.0 ** 97 * scale[:, None]
    return torch.where(b == 255, torch.full_like(v, math.nan), v).reshape(-1)[: code.numel()]


def _half_words(n, seed, tensor, step, device):
    """16 random bits for each of n elements"""
    e = torch.arange(-(-n // 8), device=device, dtype=torch.int64)
    c = [e & M32, e >> 32, torch.full_like(e, tensor), torch.full_like(e, step & M32)]
    k0, k1 = seed & M32, (seed >> 32) & M32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57          # (the wrapped 64 bits hold both 32-bit halves)
        c = [((p1 >> 32) & M32) ^ c[1] ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c[3] ^ k1, p0 & M32]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return torch.stack([w >> sh & 0xFFFF for w in c for sh in (0, 16)], 1).reshape(-1)[:n]


def _moved(p, g, m, v, step):
    """p, m and v after the step, in the type that they come in"""
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    bc1, bc2 = 1.0 - BETA1 ** step, 1.0 - BETA2 ** step
    return p * (1.0 - LR * DECAY) - (LR / bc1) * m / (torch.sqrt(v) * (1.0 / math.sqrt(bc2)) + EPS), m, v


def _adamw_plain(s, case):
    s.step += 1
    ms, vs = [], []
    for i, n in enumerate(s.sizes):
        eight = case["bits"] == 8
        m = _decode_m(s.m[i], s.m_scale[i]) if eight else s.m[i]
        v = _decode_v(s.v[i], s.v_scale[i]) if eight else s.v[i]
        p, m, v = _moved(s.p[i], s.g[i].float(), m, v, s.step)
        s.p[i].copy_(p)
        if s.shadow is not None:
            s.shadow[i].copy_(p)
        if not eight:
            s.m[i].copy_(m)
            s.v[i].copy_(v)
            continue
        for (code, scale), to, to_scale in ((_encode_m(m), s.m[i], s.m_scale[i]),
                                            (_encode_v(v, _half_words(n, s.seed, i, s.step, v.device)), s.v[i], s.v_scale[i])):
            to.copy_(code)
            to_scale.copy_(scale)
        # (four bits and a power of two: bf16 holds what the codes stand for)
        ms.append(_decode_m(s.m[i], s.m_scale[i]).to(torch.bfloat16))
        vs.append(_decode_v(s.v[i], s.v_scale[i]).to(torch.bfloat16))
    return _adamw_outputs(s, *((s.m, s.v) if case["bits"] == 32 else (ms, vs)))


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "ffn":
        return _ffn_exact(s, case)
    if case["op"] == "norm":
        return _norm_exact(s, case)
    return _adamw_exact(s, case)


def _ffn_exact(s, case):
    """Products in 64 bits; the gradients by differentiation of <dy, Y> instead of the formulas above."""
    F = case["f"]
    x, wgu, wd = s.x.double(), s.w_gate_up.double(), s.w_down.double()
    act = {"silu": torch.nn.functional.silu, "relu": torch.relu, "gelu": torch.nn.functional.gelu}[case["act"]]
    if case["way"] != "backward":
        gu = torch.einsum("rd,fd->rf", x, wgu)
        y = torch.einsum("rf,df->rd", act(gu[:, :F]) * gu[:, F:], wd)
        return {"y": y} if case["way"] == "answer" else {"y": y, "gu": gu}
    # (the pass starts from the kept GU: its gradient first, then through the product)
    gu = s.gu.double().requires_grad_()
    h = act(gu[:, :F]) * gu[:, F:]
    dy = s.dy.double()
    (dgu,) = torch.autograd.grad(h, gu, torch.einsum("rd,df->rf", dy, wd))
    return {"dx": torch.einsum("rf,fd->rd", dgu, wgu), "dw_gate_up": torch.einsum("rf,rd->fd", dgu, x),
            "dw_down": torch.einsum("rd,rf->df", dy, h.detach())}


def _norm_exact(s, case):
    """The forward formulas row by row in 64 bits; the gradients by differentiation."""
    R, D, G = case["rows"], case["d"], case["groups"]
    names = ["x", "f", "w_pre", "w_post", "gate", "scale"]
    back = case["way"] == "backward"
    a = {k: None if getattr(s, k) is None else getattr(s, k).double().requires_grad_(back) for k in names}

    def hat(v):
        if case["kind"] == "layer":
            var, mean = torch.var_mean(v, 1, unbiased=False, keepdim=True)
            return (v - mean) / (var + NORM_EPS).sqrt()
        return v / (v.pow(2).sum(1, keepdim=True) / D + NORM_EPS).sqrt()

    y = a["x"]
    if case["post"]:
        p = a["w_post"] * hat(a["f"])
        if G:
            p = p * a["gate"].repeat_interleave(R // G, 0)
        y = p + (y if a["scale"] is None else a["scale"] * y)
    n = a["w_pre"] * hat(y) if case["pre"] else None
    if not back:
        return {"y": y if case["post"] else None, "n": n}
    loss = (y * s.dy.double()).sum() + (0 if n is None else (n * s.dn.double()).sum())
    leaves = [k for k in names if a[k] is not None]
    grads = dict(zip(leaves, torch.autograd.grad(loss, [a[k] for k in leaves])))
    to = {"x": "dx", "f": "df", "w_pre": "dw_pre", "w_post": "dw_post", "gate": "dgate", "scale": "dscale"}
    return {to[k]: grads.get(k) for k in names}


def _adamw_exact(s, case):
    """32-bit states: the formulas in 64 bits.  8-bit states: the codes of the moments that 64 bits give."""
    t = s.step + 1
    ps, ms, vs = [], [], []
    for i, n in enumerate(s.sizes):
        g, p = s.g[i].double(), s.p[i].double()
        if case["bits"] == 32:
            m, v = s.m[i].double(), s.v[i].double()
        else:
            block = torch.arange(n, device=p.device) // BLOCK
            m = s.m[i].double() * s.m_scale[i].double()[block]
            code = s.v[i].to(torch.int64)
            e, f = code >> 3, (code & 7).double()
            unit = torch.where(e > 0, (8.0 + f) * 0.125 * torch.exp2((e - 30).double()), f * 0.125 * 2.0 ** -29)
            v = unit * s.v_scale[i].double()[block]
        m = m + (g - m) * (1.0 - BETA1)
        v = v + (g.square() - v) * (1.0 - BETA2)
        ps.append(p - LR * (DECAY * p + m / (1.0 - BETA1 ** t) / ((v / (1.0 - BETA2 ** t)).sqrt() + EPS)))
        if case["bits"] == 8:
            pad = -n % BLOCK
            m, v = (torch.nn.functional.pad(a, (0, pad)).view(-1, BLOCK) for a in (m, v))
            half = torch.nn.functional.pad(_half_words(n, s.seed, i, t, p.device), (0, pad)).view(-1, BLOCK).double()
            top = lambda a: torch.exp2(torch.floor(torch.log2(a.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100))))  # noqa: E731
            # e4m3 to nearest, ties to even: 3 bits behind the leading one, of 2^-6 at least
            sm, sv = top(m) / 128.0, top(v)
            q = m / sm
            ulp = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3.0)
            m = torch.round(q / ulp) * ulp * sm
            # up or down by chance
            q = v / sv
            ulp = torch.exp2(torch.floor(torch.log2(q.clamp(min=2.0 ** -29))) - 3.0)
            v = torch.floor(q / ulp + half / 65536.0) * ulp * sv
            m, v = m.reshape(-1)[:n], v.reshape(-1)[:n]
        ms.append(m)
        vs.append(v)
    pick = sorted(range(len(s.sizes)), key=lambda i: -s.sizes[i])[:12]
    out = {"p": [ps[i] for i in pick], "m": [ms[i] for i in pick], "v": [vs[i] for i in pick]}
    if s.shadow is not None:
        out["shadow"] = out["p"]
    return out
