"""Dense layers in 8-bit integers and the optimiser step over many tensors: the calls a user makes of them, and their plain forms.

A case is a plain dict.  Its "op" is one of
  linear     y = act(x W^T + b) with W in 8-bit integers (a scale for each output channel) and the tokens of x brought to 8-bit integers
             within the call (a scale for each token)
  backward   dx, dw, db of such a layer from x, the float weights, dy and (with ReLU) y: both products in 8-bit integers, each operand with
             a scale for each row of the product it enters
  adamw      one AdamW step over a list of tensors, clipped by their gradients' norm, the states in 32 bits or in 8

`own` false: elementary torch operations in float32.  `own` true: the library's entry points.
"""
import math

import torch

own = False

BLOCK = 256                    # values of a tensor that share a scale of an 8-bit state
TINY = 2.0 ** -100             # a block whose largest value lies below this holds zeros
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
STEP = 100                     # optimiser steps taken so far, this one included

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------- cases
def _linear(name, m, k, n, x="bf16", y="bf16", bias=True, relu=False, columns=False):
    return dict(name=name, op="linear", m=m, k=k, n=n, x=x, y=y, bias=bias, relu=relu, columns=columns)


def _backward(name, m, k, n, x="bf16", w="f32", dy="bf16", relu=False, columns=False):
    return dict(name=name, op="backward", m=m, k=k, n=n, x=x, w=w, dy=dy, relu=relu, columns=columns)


def _heads(name, clients, bits, grad="f32", clip=False, c_in=256, c1=128, c2=128, classes=19):
    return dict(name=name, op="adamw", what="heads", clients=clients, c_in=c_in, c1=c1, c2=c2, classes=classes, bits=bits,
                param="f32", grad=grad, copy=False, clip=clip)


def _blocks(name, layers, d, f, bits, param="f32", grad="bf16", copy=False, clip=False):
    return dict(name=name, op="adamw", what="blocks", layers=layers, d=d, f=f, bits=bits, param=param, grad=grad, copy=copy, clip=clip)


def listed():
    return [
        # one token of a served layer: the weights are read once and little else counts
        _linear("one token", 1, 2048, 5632),
        # a handful of requests that decode together
        _linear("12 tokens", 12, 4096, 4096),
        # a ragged batch through a layer of odd sizes, float32 in and out
        _linear("ragged", 333, 1000, 1003, x="f32", y="f32"),
        # a 1x1 layer with ReLU on every cell of a 1280x720 frame's feature map (90 x 160 cells, 256 -> 128 channels)
        _linear("cells 720p", 14400, 256, 128, relu=True),
        # a large batch through a wide layer: matrix-core work
        _linear("wide", 8192, 4096, 14336),
        # training a small layer of odd sizes on few tokens: launches and latency
        _backward("small backward", 480, 200, 136, x="f32", dy="f32"),
        # training the 1x1 layer on a frame's cells, its gradient channel by channel as a feature map's gradient comes
        _backward("cells backward", 14400, 256, 128, dy="f32", columns=True),
        # training a wide layer with ReLU on a large batch
        _backward("wide backward", 8192, 4096, 4096, w="bf16", relu=True),
        # one client's head, six tensors, clipped, states in 32 bits
        _heads("one head", 1, 32, clip=True),
        # two dozen clients' heads in one call, states in 8 bits
        _heads("24 heads", 24, 8),
        # layers of odd widths with bfloat16 gradients and operand copies, states in 32 bits, clipped
        _blocks("odd blocks", 12, 1000, 2731, 32, copy=True, clip=True),
        # a large model's layers, states in 8 bits
        _blocks("large blocks", 16, 2048, 5632, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {c["op"]: max((work(x) for x in listed() if x["op"] == c["op"]), key=lambda w: w["flops"]) for c in listed()}
    op = rng.choice(["linear", "linear", "backward", "adamw"])
    while True:
        if op == "linear":
            m = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 500), _log_int(rng, 500, 15000)])
            c = _linear("", m, _log_int(rng, 128, 8192), _log_int(rng, 96, 14336), x=rng.choice(["bf16", "bf16", "f32"]),
                        y=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.5, relu=rng.random() < 0.3, columns=rng.random() < 0.2)
        elif op == "backward":
            c = _backward("", _log_int(rng, 64, 15000), _log_int(rng, 96, 4096), _log_int(rng, 96, 4096), x=rng.choice(["bf16", "f32"]),
                          w=rng.choice(["f32", "bf16"]), dy=rng.choice(["f32", "bf16"]), relu=rng.random() < 0.4, columns=rng.random() < 0.3)
        elif rng.random() < 0.5:
            bits = rng.choice([8, 32])
            c = _heads("", _log_int(rng, 1, 64), bits, grad=rng.choice(["f32", "bf16"]), clip=bits == 32 and rng.random() < 0.5,
                       c_in=rng.choice([96, 256, 320]), c1=rng.choice([48, 128, 256]), c2=rng.choice([48, 128, 256]), classes=rng.randint(2, 32))
        else:
            bits = rng.choice([8, 32])
            d = _log_int(rng, 100, 2048)
            c = _blocks("", rng.randint(1, 16), d, int(d * rng.uniform(1.5, 4)), bits, param=rng.choice(["f32", "bf16"]),
                        grad=rng.choice(["f32", "bf16"]), clip=bits == 32 and rng.random() < 0.5)
            c["copy"] = c["param"] == "f32" and rng.random() < 0.5
        c.pop("name")
        w = work(c)
        if w["flops"] <= top[op]["flops"] and w["bytes"] <= top[op]["bytes"]:
            return c


def _sizes(case):
    """(values, weight decay) of each tensor of an optimiser case: matrices decay, biases and gains do not."""
    if case["what"] == "heads":
        a, b, c, n = case["c_in"], case["c1"], case["c2"], case["classes"]
        return [(9 * a * b, DECAY), (b, 0.0), (9 * b * c, DECAY), (c, 0.0), (c * n, DECAY), (n, 0.0)] * case["clients"]
    d, f = case["d"], case["f"]
    return [(d, 0.0), (d * d, DECAY), (d, 0.0), (d * f, DECAY), (f, 0.0), (f * d, DECAY)] * case["layers"]


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "adamw":
        n = sum(s for s, _ in _sizes(case))
        state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK + 8.0    # the 8-bit states' values come back as float32
        each = 2 * size[case["param"]] + size[case["grad"]] + state + (2 if case["copy"] else 0)
        return {"bytes": n * each, "flops": 16.0 * n}
    m, k, n = case["m"], case["k"], case["n"]
    if case["op"] == "linear":
        return {"bytes": m * k * size[case["x"]] + n * k + 4.0 * n * (2 if case["bias"] else 1) + m * n * size[case["y"]], "flops": 2.0 * m * n * k}
    return {"bytes": 2.0 * m * k * size[case["x"]] + m * n * size[case["dy"]] * (2 if case["relu"] else 1) + n * k * (size[case["w"]] + 4.0) + 4.0 * n, "flops": 4.0 * m * n * k}


# --------------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(m, k, g):
    """Normal values whose channels differ in size, a few of them by far, as activations' do."""
    size = torch.exp(0.5 * torch.randn(k, device="cuda", generator=g))
    size[torch.rand(k, device="cuda", generator=g) < 0.004] *= 12.0
    return torch.randn(m, k, device="cuda", generator=g) * size


def _pad16(k):
    return (k + 15) // 16 * 16


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, g)
    m, k, n = case["m"], case["k"], case["n"]
    s = dict(case)
    x = _activations(m, k, g).to(_DTYPE[case["x"]])
    w = torch.randn(n, k, device="cuda", generator=g) / math.sqrt(k)
    if case["op"] == "linear":
        q, scale = _quantize(w)
        s["wq"] = torch.zeros(n, _pad16(k), dtype=torch.int8, device="cuda")
        s["wq"][:, :k] = q.to(torch.int8)
        s["scale"] = scale.reshape(n)
        s["bias"] = torch.randn(n, device="cuda", generator=g) if case["bias"] else None
        s["x"] = x.t().contiguous().t() if case["columns"] else x
        s["out"] = torch.empty(m, n, dtype=_DTYPE[case["y"]], device="cuda")
        if own:
            s["workspace"] = _library().new_int8_workspace(m, n, k)
        return s
    s["x"], s["w"] = x, w.to(_DTYPE[case["w"]])
    dy = (1e-3 * torch.randn(m, n, device="cuda", generator=g) * torch.exp(torch.randn(m, 1, device="cuda", generator=g))).to(_DTYPE[case["dy"]])
    s["y"] = torch.relu(torch.randn(m, n, device="cuda", generator=g)).to(_DTYPE[case["dy"]]) if case["relu"] else None
    s["dy"] = dy
    if case["columns"]:
        s["dy"] = dy.t().contiguous().t()
        s["y"] = None if s["y"] is None else s["y"].t().contiguous().t()
    s["dx"] = torch.empty(m, k, dtype=_DTYPE[case["x"]], device="cuda")
    s["dw"] = torch.empty(n, k, device="cuda")
    s["db"] = torch.empty(n, device="cuda")
    if own:
        s["workspace"] = _library().new_int8_workspace(m, n, k, backward=True)
    return s


def _prepare_adamw(case, g):
    """One buffer for each kind of value, every tensor at a multiple of BLOCK with zeros behind it."""
    sizes = _sizes(case)
    starts, at = [], 0
    for n, _ in sizes:
        starts.append(at)
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    blocks = at // BLOCK
    decay = torch.tensor([d for _, d in sizes], device="cuda")
    per = torch.tensor([(n + BLOCK - 1) // BLOCK for n, _ in sizes], device="cuda")
    s = dict(case, decay=torch.repeat_interleave(decay, per)[:, None])
    size = torch.repeat_interleave(torch.exp(torch.randn(len(sizes), device="cuda", generator=g)), per)[:, None]
    grad = 1e-4 * size * torch.randn(blocks, BLOCK, device="cuda", generator=g)
    m = 3e-5 * size * torch.randn(blocks, BLOCK, device="cuda", generator=g)
    u = 1e-4 * size * (0.2 + torch.rand(blocks, BLOCK, device="cuda", generator=g))
    p = 0.02 * torch.randn(blocks, BLOCK, device="cuda", generator=g)
    for t in (grad, m, u, p):
        flat = t.view(-1)
        for (n, _), b in zip(sizes, starts):
            if n % BLOCK:
                flat[b + n:(b + n + BLOCK - 1) // BLOCK * BLOCK] = 0
    s["p"], s["g"] = p.to(_DTYPE[case["param"]]), grad.to(_DTYPE[case["grad"]])
    del p, grad
    s["copy16"] = torch.zeros(blocks, BLOCK, dtype=torch.bfloat16, device="cuda") if case["copy"] else None
    if case["bits"] == 32:
        s["m"], s["v"] = m, u * u
    else:
        s["m"], s["m_scale"], s["v"], s["v_scale"] = _encode(m, u)
        s["m_out"], s["v_out"] = (torch.empty(blocks, BLOCK, device="cuda") for _ in range(2))
    s["norm"] = torch.empty(1, device="cuda")
    # clipped: to about a third of the norm; otherwise a limit that ordinary gradients keep
    s["max_norm"] = 3e-5 * math.sqrt(at) if case["clip"] else 1e6
    if own:
        st = _library()

        def views(t):
            return [t.view(-1)[b:b + n] for (n, _), b in zip(sizes, starts)]

        def scales(t):
            return [t.view(-1)[b // BLOCK:b // BLOCK + (n + BLOCK - 1) // BLOCK] for (n, _), b in zip(sizes, starts)]

        s["tensors"] = st.AdamWTensors(views(s["p"]), views(s["g"]), views(s["m"]), views(s["v"]),
                                       m_scales=scales(s["m_scale"]) if case["bits"] == 8 else None,
                                       v_scales=scales(s["v_scale"]) if case["bits"] == 8 else None,
                                       copies=views(s["copy16"]) if case["copy"] else None,
                                       weight_decay=[d for _, d in sizes])
        s["workspace"] = st.new_adamw_workspace(s["tensors"])
    return s


def _library():
    import paper_2003_10735_amd
    return paper_2003_10735_amd


# -------------------------------------------------------------------------------------------------------------- a pass
def run(s):
    if s["op"] == "linear":
        return _run_linear(s)
    return _run_backward(s) if s["op"] == "backward" else _run_adamw(s)


def _quantize(x):
    """Rows of x as whole numbers of -127 .. 127 (held as float32) and a scale for each row [rows, 1]."""
    x = x.float()
    top = x.abs().amax(dim=1, keepdim=True)
    r = torch.where(top > 0, 127.0 / top, torch.zeros_like(top))
    return torch.round(x * r), top / 127.0


def _run_linear(s):
    if own:
        return _library().st_int8_linear(s["x"], s["wq"], s["scale"], bias=s["bias"], relu=s["relu"], out=s["out"], workspace=s["workspace"])
    q, scale = _quantize(s["x"])
    y = torch.mm(q, s["wq"][:, :s["k"]].float().t()) * scale * s["scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["relu"]:
        y = torch.relu(y)
    return y.to(_DTYPE[s["y"]])


def _run_backward(s):
    if own:
        return _library().st_int8_linear_backward(s["x"], s["w"], s["dy"], y=s["y"], dx=s["dx"], dw=s["dw"], db=s["db"], workspace=s["workspace"])
    dz = s["dy"].float()
    if s["y"] is not None:
        dz = torch.where(s["y"] > 0, dz, torch.zeros_like(dz))
    a, a_scale = _quantize(dz)
    b, b_scale = _quantize(s["w"].t())
    dx = torch.mm(a, b.t()) * a_scale * b_scale.t()
    a, a_scale = _quantize(dz.t())
    b, b_scale = _quantize(s["x"].t())
    dw = torch.mm(a, b.t()) * a_scale * b_scale.t()
    return dx.to(s["x"].dtype), dw, dz.sum(dim=0)


def _decode(qm, m_scale, qv, v_scale):
    qm, qv = qm.float(), qv.float()
    return qm * qm.abs() * m_scale, qv * qv * v_scale


def _encode(m, u):
    """Codes and scales [blocks, 1] of m and of u = sqrt(v): a code stands for its square times the block's scale."""
    top = m.abs().amax(dim=1, keepdim=True)
    some = top >= TINY
    m_scale = torch.where(some, top / 16129.0, torch.zeros_like(top))
    r = torch.where(some, 16129.0 / top, torch.zeros_like(top))
    qm = (torch.round(torch.sqrt(m.abs() * r)) * torch.sign(m)).to(torch.int8)
    top = u.amax(dim=1, keepdim=True)
    some = top >= TINY
    v_scale = torch.where(some, top / 65025.0, torch.zeros_like(top))
    r = torch.where(some, 65025.0 / top, torch.zeros_like(top))
    qv = torch.round(torch.sqrt(u * r))
    qv = torch.where((u > 0) & some, torch.clamp(qv, min=1.0), qv).to(torch.uint8)
    return qm, m_scale, qv, v_scale


def _run_adamw(s):
    eight = s["bits"] == 8
    if own:
        st = _library()
        st.st_adamw_step(s["tensors"], STEP, LR, beta1=BETA1, beta2=BETA2, eps=EPS, max_norm=s["max_norm"], grad_norm=s["norm"],
                         workspace=s["workspace"])
        if eight:
            st.st_adamw_state(s["m"], s["m_scale"], s["v"], s["v_scale"], m_out=s["m_out"], v_out=s["v_out"])
    else:
        g = s["g"].float()
        norm = torch.sqrt((g * g).sum())
        s["norm"].copy_(norm)
        g = g * torch.clamp(s["max_norm"] / norm, max=1.0)
        if eight:
            m, u = _decode(s["m"], s["m_scale"], s["v"], s["v_scale"])
            v = u * u
        else:
            m, v = s["m"], s["v"]
        m = m * BETA1 + g * (1 - BETA1)
        v = v * BETA2 + g * g * (1 - BETA2)
        del g
        u = torch.sqrt(v)
        p = s["p"].float() * (1 - LR * s["decay"]) - LR / (1 - BETA1 ** STEP) * (m / (u * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS))
        s["p"].copy_(p)
        if s["copy"]:
            s["copy16"].copy_(p)
        del p
        if eight:
            del v
            for name, value in zip(("m", "m_scale", "v", "v_scale"), _encode(m, u)):
                s[name].copy_(value)
            m, u = _decode(s["m"], s["m_scale"], s["v"], s["v_scale"])
            s["m_out"].copy_(m)
            s["v_out"].copy_(u * u)
        else:
            s["m"].copy_(m)
            s["v"].copy_(v)
    out = {"p": s["p"], "norm": s["norm"], "m": s["m_out"] if eight else s["m"], "v": s["v_out"] if eight else s["v"]}
    if s["copy"]:
        out["copy"] = s["copy16"]
    return out


# ----------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        x = s["x"].double()
        a = x.abs().max(dim=1).values
        qx = torch.where(a[:, None] > 0, torch.round(x / a[:, None] * 127), 0.0)
        w = s["wq"].double()[:, :case["k"]] * s["scale"].double()[:, None]
        y = (qx * (a / 127)[:, None]) @ w.t().contiguous()
        if s["bias"] is not None:
            y += s["bias"].double()
        return y.clamp_(min=0) if case["relu"] else y
    if case["op"] == "backward":
        dz = s["dy"].double()
        if s["y"] is not None:
            dz = dz * (s["y"].double() > 0)

        def on_grid(t, dim):
            a = t.abs().max(dim=dim, keepdim=True).values
            return torch.where(a > 0, torch.round(t / a * 127) * a / 127, 0.0)

        dx = on_grid(dz, 1) @ on_grid(s["w"].double(), 0)
        dw = on_grid(dz, 0).t().contiguous() @ on_grid(s["x"].double(), 0)
        return dx, dw, dz.sum(0)
    g, p = s["g"].double(), s["p"].double()
    norm = g.square().sum().sqrt()
    g *= min(1.0, s["max_norm"] / norm.item())
    if case["bits"] == 8:
        m = s["m"].double().abs() * s["m"].double() * s["m_scale"].double()
        v = (s["v"].double().square() * s["v_scale"].double()).square()
    else:
        m, v = s["m"].double(), s["v"].double()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g.square()
    del g
    p = p - LR * s["decay"].double() * p - LR * (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    if case["bits"] == 8:
        a = m.abs().max(dim=1, keepdim=True).values
        q = torch.where(a > 0, torch.round(127 * (m.abs() / a).sqrt()) / 127, 0.0)
        m = torch.sign(m) * q.square() * a
        u = v.sqrt()
        a = u.max(dim=1, keepdim=True).values
        q = torch.where(a > 0, torch.round(255 * (u / a).sqrt()) / 255, 0.0)
        q = torch.where(u > 0, q.clamp(min=1 / 255), q)
        v = (q.square() * a).square()
    out = {"p": p, "norm": norm.reshape(1), "m": m, "v": v}
    if case["copy"]:
        out["copy"] = p
    return out
