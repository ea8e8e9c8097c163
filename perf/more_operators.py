"""Dense layers in bfloat16 or float32 with bias, activation and residual, their gradients, and the norm and clipping of many gradients: the
calls a user makes of them, and their plain forms.

A case is a plain dict.  Its "op" is one of
  linear     y = act(x W^T + b) + r, and where the layer is being trained z = x W^T + b beside it
  backward   dx, dw, db of such a layer from x, W, dy and z
  clip       the 2-norm of all gradients of a list, and the gradients themselves, clipped by it, in the type that the optimiser's list takes

`own` false: elementary torch operations in float32.  `own` true: the library's entry points.
"""
import math

import torch

own = False

BLOCK = 64                     # values that a tensor of a list begins at a multiple of
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2, None: 0}
_ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


# ---------------------------------------------------------------------------------------------------------------- cases
def _linear(name, m, k, n, dtype="bf16", y="bf16", act="none", bias=True, residual=None, pre=False, x_columns=False, w_columns=False):
    return dict(name=name, op="linear", m=m, k=k, n=n, dtype=dtype, y=y, act=act, bias=bias, residual=residual, pre=pre,
                x_columns=x_columns, w_columns=w_columns)


def _backward(name, m, k, n, dtype="bf16", dy="bf16", dw="bf16", act="none", dy_columns=False, w_columns=False):
    return dict(name=name, op="backward", m=m, k=k, n=n, dtype=dtype, dy=dy, dw=dw, act=act, dy_columns=dy_columns, w_columns=w_columns)


def _heads(name, clients, out=None, scale=1.0, c_in=256, c1=128, c2=128, classes=19):
    return dict(name=name, op="clip", what="heads", clients=clients, c_in=c_in, c1=c1, c2=c2, classes=classes, matrices="f32", vectors="f32",
                out=out, scale=scale)


def _blocks(name, layers, d, f, matrices="bf16", vectors="f32", out=None, scale=1.0):
    return dict(name=name, op="clip", what="blocks", layers=layers, d=d, f=f, matrices=matrices, vectors=vectors, out=out, scale=scale)


def listed():
    return [
        # one token of a served layer: the weights are read once and little else counts
        _linear("one token", 1, 2048, 5632, act="silu"),
        # a handful of requests that decode together, back to the residual stream
        _linear("12 tokens", 12, 4096, 4096, residual="bf16"),
        # a ragged batch through a float32 layer of odd sizes
        _linear("ragged", 333, 1000, 1003, dtype="f32", y="f32", act="gelu"),
        # a 1x1 layer with ReLU on every cell of a 1280x720 frame's feature map (90 x 160 cells, 256 -> 128 channels)
        _linear("cells 720p", 14400, 256, 128, act="relu"),
        # the wide layer of a block in training, which keeps what its activation was given
        _linear("wide", 8192, 4096, 14336, act="gelu_tanh", pre=True),
        # training a small float32 layer of odd sizes on few tokens: launches and latency
        _backward("small backward", 480, 200, 136, dtype="f32", dy="f32", dw="f32", act="gelu"),
        # training the 1x1 layer on a frame's cells, its gradient in float32 and channel by channel as a feature map's gradient comes
        _backward("cells backward", 14400, 256, 128, dy="f32", act="relu", dy_columns=True),
        # training a wide layer on a large batch
        _backward("wide backward", 8192, 4096, 4096, act="silu"),
        # one client's head, six tensors
        _heads("one head", 1),
        # layers of odd widths, matrices in bfloat16 and vectors in float32, into the one type that the optimiser's list takes, a loss scale taken out
        _blocks("odd blocks", 12, 1000, 2731, out="f32", scale=2.0 ** -10),
        # a large model's layers
        _blocks("large blocks", 16, 2048, 5632, vectors="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {op: max((work(x) for x in listed() if x["op"] == op), key=lambda w: w["flops"]) for op in ("linear", "backward", "clip")}
    op = rng.choice(["linear", "linear", "linear", "backward", "backward", "clip"])
    while True:
        if op == "linear":
            m = rng.choice([1, rng.randint(2, 32), _log_int(rng, 33, 500), _log_int(rng, 500, 15000)])
            c = _linear("", m, _log_int(rng, 96, 8192), _log_int(rng, 96, 14336), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                        y=rng.choice(["bf16", "f32"]), act=rng.choice(_ACTS), bias=rng.random() < 0.6, residual=rng.choice([None, None, "bf16", "f32"]),
                        pre=rng.random() < 0.3, x_columns=rng.random() < 0.15, w_columns=rng.random() < 0.25)
        elif op == "backward":
            dtype, act = rng.choice(["bf16", "bf16", "f32"]), rng.choice(_ACTS)
            dy = rng.choice(["f32", "bf16"])
            # (bfloat16 operands: what the activation or float32 leaves of dy is rounded to bfloat16, and weights' gradients are asked for in it)
            exact_operands = dtype == "f32" or (dy == "bf16" and act in ("none", "relu"))
            c = _backward("", _log_int(rng, 16, 15000), _log_int(rng, 96, 4096), _log_int(rng, 96, 8192), dtype=dtype, dy=dy,
                          dw="f32" if exact_operands and rng.random() < 0.7 else "bf16", act=act, dy_columns=rng.random() < 0.25,
                          w_columns=rng.random() < 0.2)
        else:
            out = rng.choice([None, "f32", "bf16"])
            scale = rng.choice([1.0, 2.0 ** -10])
            if rng.random() < 0.4:
                c = _heads("", _log_int(rng, 1, 64), out=out, scale=scale, c_in=rng.choice([96, 256, 320]), c1=rng.choice([48, 128, 256]),
                           c2=rng.choice([48, 128, 256]), classes=rng.randint(2, 32))
            else:
                d = _log_int(rng, 100, 2048)
                c = _blocks("", rng.randint(1, 16), d, int(d * rng.uniform(1.5, 4)), matrices=rng.choice(["f32", "bf16"]),
                            vectors=rng.choice(["f32", "bf16"]), out=out, scale=scale)
        c.pop("name")
        w = work(c)
        if w["flops"] <= top[op]["flops"] and w["bytes"] <= top[op]["bytes"] and (op == "clip" or c["dtype"] == "bf16" or w["flops"] <= top[op]["flops"] / 4):
            return c


def _sizes(case):
    """(matrices, vectors): values of each tensor of a list."""
    if case["what"] == "heads":
        a, b, c, n = case["c_in"], case["c1"], case["c2"], case["classes"]
        return [9 * a * b, 9 * b * c, c * n] * case["clients"], [b, c, n] * case["clients"]
    d, f = case["d"], case["f"]
    return [d * d, d * f, f * d] * case["layers"], [d, d, f] * case["layers"]


def work(case):
    if case["op"] == "clip":
        total, bytes_ = 0, 0
        for sizes, kind in zip(_sizes(case), ("matrices", "vectors")):
            total += sum(sizes)
            bytes_ += sum(sizes) * (_BYTES[case[kind]] + _BYTES[case["out"] or case[kind]])
        return {"bytes": float(bytes_), "flops": 3.0 * total}
    m, k, n = case["m"], case["k"], case["n"]
    e = _BYTES[case["dtype"]]
    if case["op"] == "linear":
        return {"bytes": float((m * k + n * k) * e + (4 * n if case["bias"] else 0) + m * n * (_BYTES[case["y"]] * (2 if case["pre"] else 1) + _BYTES[case["residual"]])),
                "flops": 2.0 * m * n * k}
    return {"bytes": float(2 * (m * k + n * k) * e + n * k * (_BYTES[case["dw"]] - e) + m * n * (_BYTES[case["dy"]] + (0 if case["act"] == "none" else e)) + 4 * n),
            "flops": 4.0 * m * n * k}


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


def _laid(t, columns):
    return t.t().contiguous().t() if columns else t


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "clip":
        return _prepare_clip(case, g)
    m, k, n = case["m"], case["k"], case["n"]
    dtype = _DTYPE[case["dtype"]]
    s = dict(case)
    x = _activations(m, k, g)
    # outputs of about one, whatever the inputs' channels: some activations then saturate and some do not
    w = torch.randn(n, k, device="cuda", generator=g) / (x.square().mean() * k).sqrt()
    s["w"] = _laid(w.to(dtype), case["w_columns"])
    if case["op"] == "linear":
        s["x"] = _laid(x.to(dtype), case["x_columns"])
        s["b"] = 0.5 * torch.randn(n, device="cuda", generator=g) if case["bias"] else None
        s["r"] = torch.randn(m, n, device="cuda", generator=g).to(_DTYPE[case["residual"]]) if case["residual"] else None
        s["out"] = torch.empty(m, n, dtype=_DTYPE[case["y"]], device="cuda")
        s["z"] = torch.empty(m, n, dtype=_DTYPE[case["y"]], device="cuda") if case["pre"] else None
    else:
        s["x"] = x.to(dtype)
        dy = 1e-3 * torch.randn(m, n, device="cuda", generator=g) * torch.exp(torch.randn(m, 1, device="cuda", generator=g))
        s["dy"] = _laid(dy.to(_DTYPE[case["dy"]]), case["dy_columns"])
        s["z"] = None if case["act"] == "none" else torch.randn(m, n, device="cuda", generator=g).to(dtype)
        s["dx"] = torch.empty(m, k, dtype=dtype, device="cuda")
        s["dw"] = torch.empty(n, k, dtype=_DTYPE[case["dw"]], device="cuda")
        s["db"] = torch.empty(n, device="cuda")
    if own:
        st = _library()
        s["activation"] = [st.ST_ACT_NONE, st.ST_ACT_RELU, st.ST_ACT_GELU, st.ST_ACT_GELU_TANH, st.ST_ACT_SILU][_ACTS.index(case["act"])]
        if case["op"] == "linear":
            s["workspace"] = st.new_linear_workspace(s["x"], s["w"])
        else:
            s["workspace"] = st.new_linear_workspace(s["x"], s["w"], s["dy"], s["activation"])
    return s


def _prepare_clip(case, g):
    """One buffer for each kind of tensor, every tensor at a multiple of BLOCK with zeros behind it."""
    s = dict(case)
    views, outs, total = [], [], 0
    for sizes, kind in zip(_sizes(case), ("matrices", "vectors")):
        starts, at = [], 0
        for n in sizes:
            starts.append(at)
            at += (n + BLOCK - 1) // BLOCK * BLOCK
        per = torch.tensor([(n + BLOCK - 1) // BLOCK for n in sizes], device="cuda")
        size = torch.repeat_interleave(torch.exp(torch.randn(len(sizes), device="cuda", generator=g)), per)[:, None]
        t = (1e-4 / case["scale"]) * size * torch.randn(at // BLOCK, BLOCK, device="cuda", generator=g)
        flat = t.view(-1)
        for n, b in zip(sizes, starts):
            flat[b + n:b + (n + BLOCK - 1) // BLOCK * BLOCK] = 0
        s[kind] = t.to(_DTYPE[case[kind]])
        s[kind + "_out"] = torch.zeros(at // BLOCK, BLOCK, dtype=_DTYPE[case["out"] or case[kind]], device="cuda")
        views += [s[kind].view(-1)[b:b + n] for n, b in zip(sizes, starts)]
        outs += [s[kind + "_out"].view(-1)[b:b + n] for n, b in zip(sizes, starts)]
        total += at
    s["norm"] = torch.empty(1, device="cuda")
    s["max_norm"] = 3e-5 * math.sqrt(total)      # about a third of the norm
    if own:
        st = _library()
        s["tensors"] = st.GradTensors(views, outs)
        s["workspace"] = st.new_grad_workspace(s["tensors"])
    return s


def _library():
    import paper_2003_10735_amd
    return paper_2003_10735_amd


# -------------------------------------------------------------------------------------------------------------- a pass
def run(s):
    if s["op"] == "linear":
        return _run_linear(s)
    return _run_backward(s) if s["op"] == "backward" else _run_clip(s)


def _normal(z):
    """The normal distribution function, and its density."""
    return 0.5 * torch.erfc(z * -math.sqrt(0.5)), torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _activate(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * _normal(z)[0]
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _slope(z, act):
    """The derivative of the activation at z."""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        share, density = _normal(z)
        return share + z * density
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * (math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * z * z))
    if act == "silu":
        t = torch.sigmoid(z)
        return t * (1.0 + z * (1.0 - t))
    return torch.ones_like(z)


def _run_linear(s):
    if own:
        y = _library().st_linear(s["x"], s["w"], bias=s["b"], activation=s["activation"], residual=s["r"], pre=s["z"], out=s["out"],
                                 workspace=s["workspace"])
        return {"y": y, "z": s["z"]} if s["pre"] else y
    z = torch.mm(s["x"].float(), s["w"].float().t())
    if s["b"] is not None:
        z = z + s["b"]
    y = _activate(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    y = y.to(_DTYPE[s["y"]])
    return {"y": y, "z": z.to(_DTYPE[s["y"]])} if s["pre"] else y


def _run_backward(s):
    if own:
        return _library().st_linear_backward(s["x"], s["w"], s["dy"], pre=s["z"], activation=s["activation"], dx=s["dx"], dw=s["dw"], db=s["db"],
                                             workspace=s["workspace"])
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _slope(s["z"].float(), s["act"])
    dx = torch.mm(dz, s["w"].float())
    dw = torch.mm(dz.t(), s["x"].float())
    return dx.to(s["dx"].dtype), dw.to(s["dw"].dtype), dz.sum(dim=0)


def _run_clip(s):
    if own:
        _library().st_grad_clip(s["tensors"], max_norm=s["max_norm"], grad_scale=s["scale"], grad_norm=s["norm"], workspace=s["workspace"])
    else:
        a, b = s["matrices"].float(), s["vectors"].float()
        norm = torch.sqrt(a.square().sum(dtype=torch.float64) + b.square().sum(dtype=torch.float64)).float() * s["scale"]
        c = s["scale"] * torch.clamp(s["max_norm"] / norm, max=1.0)
        s["norm"].copy_(norm)
        s["matrices_out"].copy_(a * c)
        s["vectors_out"].copy_(b * c)
    return {"norm": s["norm"], "matrices": s["matrices_out"], "vectors": s["vectors_out"]}


# ----------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    act = case["op"] != "clip" and case["act"]
    z = None
    if case["op"] == "linear":
        z = s["x"].double() @ s["w"].double().t().contiguous()
        if s["b"] is not None:
            z += s["b"].double()
    elif case["op"] == "backward" and act != "none":
        z = s["z"].double()
    c0 = math.sqrt(2.0 / math.pi)
    if case["op"] == "linear":
        if act == "relu":
            y = z.clamp(min=0)
        elif act == "gelu":
            y = z * torch.special.ndtr(z)
        elif act == "gelu_tanh":
            y = z / (1 + torch.exp(-2 * c0 * (z + 0.044715 * z ** 3)))
        elif act == "silu":
            y = z / (1 + torch.exp(-z))
        else:
            y = z.clone()
        if s["r"] is not None:
            y += s["r"].double()
        return {"y": y, "z": z} if case["pre"] else y
    if case["op"] == "backward":
        dz = s["dy"].double()
        if act == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif act == "gelu":
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi))
        elif act == "gelu_tanh":
            p = 1 / (1 + torch.exp(-2 * c0 * (z + 0.044715 * z ** 3)))
            dz = dz * (p + z * p * (1 - p) * 2 * c0 * (1 + 3 * 0.044715 * z.square()))
        elif act == "silu":
            p = 1 / (1 + torch.exp(-z))
            dz = dz * (p + z * p * (1 - p))
        dz = dz.contiguous()
        return dz @ s["w"].double().contiguous(), dz.t().contiguous() @ s["x"].double(), dz.sum(0)
    a, b = s["matrices"].double() * s["scale"], s["vectors"].double() * s["scale"]
    norm = (a.square().sum() + b.square().sum()).sqrt()
    c = min(1.0, s["max_norm"] / norm.item())
    return {"norm": norm.reshape(1), "matrices": a * c, "vectors": b * c}
