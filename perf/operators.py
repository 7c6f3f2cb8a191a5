"""Cases that measure the operators of the residual encoder's training and
serving: the linear layer with its epilogue (forward and backward), the layer
norm (forward and backward) and the 8-bit activation checkpoints.

Every pass has two forms. The plain form (`own` false) is written in
elementary torch operations in 32 bits, rounded once at the end; the other
(`own` true) makes the calls a user makes of paper_2608_15438_gb300.ops.
exact() states the same definitions in 64 bits.

Definitions, for rows x [m x k], weights w [n x k]:
  linear           z = x w^T + bias, y = act(z) + residual
  its gradients    dz = dy act'(z), dx = dz w, dw = dz^T x, dbias = sum_m dz
  layer norm       y = (x - mean) rstd weight + bias, rstd = (var + eps)^-1/2
  its gradients    xh = (x - mean) rstd, g = dy weight,
                   dx = rstd (g - mean(g) - xh mean(g xh)) + residual's gradient,
                   dweight = sum_m dy xh, dbias = sum_m dy
  checkpoint       groups of 32 columns of a row share a scale 2^e, the least
                   power of two with |v| 2^-e < 127.5 over the group; a value
                   is held as the 8-bit whole number round(v 2^-e), ties to even
"""
import math

import torch

own = False

EPS = 1e-5
GROUP = 32
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    def linear(name, m, k, n, **kw):
        c = {"name": name, "op": "linear", "dtype": "bf16", "m": m, "k": k, "n": n, "act": "none",
             "residual": False, "save": "no", "pad": 0}
        c.update(kw)
        return c

    def norm(name, op, m, k, **kw):
        c = {"name": name, "op": op, "dtype": "bf16", "m": m, "k": k, "save": False, "pad": 0,
             "residual": False, "from8": False}
        c.update(kw)
        return c

    return [
        # one query of 1536 values through the widening layer of a block: the latency of serving
        linear("linear-one-query", 1, 1536, 6144, act="gelu"),
        # a ragged layer between odd widths, its rows cut out of a wider buffer
        linear("linear-odd-widths", 1000, 771, 1013, act="relu", residual=True, pad=5),
        # the benchmark's 10,000 queries through the widening layer, keeping what a backward pass needs
        linear("linear-queries", 10000, 1536, 6144, act="gelu", save="z"),
        # base rows through the narrowing layer of a block with its residual, as an index build encodes them
        linear("linear-base-rows", 65536, 6144, 1536, residual=True),
        # gradients of the widening layer for the training mini-batch of 4096
        linear("linear-backward-minibatch", 4096, 1536, 6144, op="linear_backward", act="gelu"),
        # gradients of the 96 -> 384 layer of the 96-dimensional workload in a small batch
        linear("linear-backward-small", 1000, 96, 384, op="linear_backward", act="relu", dtype="f16"),
        # a few queries' norm while serving
        norm("norm-few-queries", "layer_norm", 64, 1536),
        # the norm over a slice of the base rows during an index build
        norm("norm-base-rows", "layer_norm", 262144, 1536),
        # the norm's gradients in a large training batch, with the gradient of the block's residual added
        norm("norm-backward-batch", "layer_norm_backward", 65536, 1536, residual=True),
        # the same in 32 bits at an odd width and batch
        norm("norm-backward-odd", "layer_norm_backward", 30011, 387, dtype="f32"),
        # the hidden activations of a large batch held in 8 bits and read back
        norm("checkpoint-batch", "checkpoint", 65536, 6144),
        # a training step of the widening layer that keeps its input and its pre-activations in 8 bits
        linear("linear-step-checkpointed", 16384, 1536, 6144, op="linear_step8", act="gelu"),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["linear", "linear", "linear_backward", "linear_backward", "linear_step8",
                     "layer_norm", "layer_norm_backward", "checkpoint"])
    pad = rng.choice([0, 0, 0, 3, 8])
    if op.startswith("linear"):
        passes = {"linear": 1, "linear_backward": 2, "linear_step8": 3}[op]
        while True:
            m, k, n = size(1, 65536), size(16, 6144), size(16, 6144)
            if rng.random() < 0.5:  # half of the layers have widths that are multiples of 32
                k, n = max(32, k // 32 * 32), max(32, n // 32 * 32)
            if m * k * n * passes <= 65536 * 6144 * 1536 and 3072 not in (m, k, n):
                break
        return {"op": op, "dtype": rng.choice(["bf16", "f16"]), "m": m, "k": k, "n": n,
                # 8-bit pre-activations serve smooth activations: a ReLU's slope is one bit of the exact value
                "act": rng.choice(["none", "gelu", "silu"] if op == "linear_step8" else ["none", "relu", "gelu", "silu"]),
                "residual": op == "linear" and rng.random() < 0.5,
                "save": rng.choice(["no", "z"]) if op == "linear" else "no", "pad": pad}
    while True:
        m, k = size(1, 262144), size(16, 8192)
        if m * k <= 262144 * 1536 and 3072 not in (m, k):
            break
    return {"op": op, "dtype": rng.choice(["bf16", "f16", "f32"]), "m": m, "k": k,
            "save": op == "layer_norm" and rng.random() < 0.5, "pad": pad,
            "residual": op == "layer_norm_backward" and rng.random() < 0.5,
            "from8": op == "layer_norm_backward" and rng.random() < 0.3}


def _rows(case, g, rows, cols, scale=1.0, shift=0.0):
    """Activations: normal values, a few columns of them much larger than the
    rest, as residual streams have; `pad` more columns in the buffer's rows."""
    dt = DTYPES[case["dtype"]]
    pitch = cols + case["pad"]
    x = torch.randn(rows, pitch, generator=g, device="cuda", dtype=torch.float32)
    amp = torch.full((pitch,), scale, device="cuda")
    amp[torch.randint(0, pitch, (max(1, pitch // 200),), generator=g, device="cuda")] = 6.0 * scale
    return x.mul_(amp).add_(shift).to(dt)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    m, k, op = case["m"], case["k"], case["op"]
    s = {"case": case, "x": _rows(case, g, m, k, 1.0, 0.1 if op.startswith("layer") else 0.0)}
    if op.startswith("linear"):
        n = case["n"]
        w = torch.randn(n, k, generator=g, device="cuda")
        s["w"] = (w / math.sqrt(k)).to(dt)
        s["bias"] = torch.randn(n, generator=g, device="cuda") * 0.1
        if op == "linear_step8":  # all of the layer's parameters in the 16-bit type
            s["bias"] = s["bias"].to(dt)
        if case["residual"]:
            s["residual"] = _rows(case, g, m, n)
        if op != "linear":
            s["dy"] = _rows(case, g, m, n, 0.01)
        if op == "linear_backward" and case["act"] != "none":
            s["z"] = (s["x"].float() @ s["w"].float().T + s["bias"]).to(dt)
    elif op.startswith("layer_norm"):
        s["weight"] = 1.0 + 0.2 * torch.randn(k, generator=g, device="cuda")
        s["bias"] = torch.randn(k, generator=g, device="cuda") * 0.1
        if op == "layer_norm_backward":
            s["dy"] = _rows(case, g, m, k, 0.01)
            if case["residual"]:
                s["dres"] = _rows(case, g, m, k, 0.01)
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + EPS)
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2608_15438_gb300 import ops

    c = s["case"]
    op = c["op"]
    if op == "linear":
        return ops.linear(s["x"], s["w"], s["bias"], act=c["act"], residual=s.get("residual"),
                          save=None if c["save"] == "no" else c["save"])
    if op == "linear_backward":
        return ops.linear_backward(s["dy"], s["x"], s["w"], z=s.get("z"), act=c["act"])
    if op == "linear_step8":
        x8 = ops.checkpoint8(s["x"])
        if c["act"] == "none":
            y, z8 = ops.linear(s["x"], s["w"], s["bias"]), None
        else:
            y, z8 = ops.linear(s["x"], s["w"], s["bias"], act=c["act"], save="z8")
        return (y,) + tuple(ops.linear_backward(s["dy"], x8, s["w"], z=z8, act=c["act"],
                                                 bias_dtype=s["bias"].dtype))
    if op == "layer_norm":
        return ops.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, save=c["save"])
    if op == "layer_norm_backward":
        x = ops.checkpoint8(s["x"]) if c["from8"] else s["x"]
        return ops.layer_norm_backward(s["dy"], x, s["weight"], s["mean"], s["rstd"],
                                       residual_grad=s.get("dres"))
    return ops.checkpoint8_read(ops.checkpoint8(s["x"]))


# ---------------------------------------------------------------- plain form, 32 bits


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.7071067811865476))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.7071067811865476)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _held8(x):
    """The values that the 8-bit checkpoint of x (fp32) stands for."""
    m, k = x.shape
    pad = -k % GROUP
    v = torch.nn.functional.pad(x, (0, pad)).view(m, -1, GROUP)
    top = v.abs().amax(2, keepdim=True).contiguous().view(torch.int32)
    e = ((top + 0x10000) >> 23).clamp(7, 254)
    up, down = ((260 - e) << 23).view(torch.float32), ((e - 6) << 23).view(torch.float32)
    q = torch.round(v * up).clamp(-127.0, 127.0)
    return (q * down).view(m, -1)[:, :k]


def _gradients(dy, x, w, z, act, types):
    dz = dy if act == "none" else dy * _act_slope(z, act)
    return (dz @ w).to(types[0]), (dz.T @ x).to(types[1]), dz.sum(0).to(types[2])


def _run_plain(s):
    c = s["case"]
    op, dt = c["op"], DTYPES[c["dtype"]]
    x = s["x"].float()
    if op.startswith("linear"):
        w = s["w"].float()
        if op == "linear_backward":
            z = s["z"].float() if "z" in s else None
            return _gradients(s["dy"].float(), x, w, z, c["act"], (dt, dt, torch.float32))
        z = x @ w.T + s["bias"].float()
        if op == "linear_step8":
            grads = _gradients(s["dy"].float(), _held8(x), w, _held8(z), c["act"], (dt, dt, dt))
            return (_act(z, c["act"]).to(dt),) + grads
        y = _act(z, c["act"])
        if c["residual"]:
            y = y + s["residual"].float()
        return (y.to(dt), z.to(dt)) if c["save"] == "z" else y.to(dt)
    if op == "checkpoint":
        return _held8(x).to(dt)
    if op == "layer_norm":
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((d * d).mean(1) + EPS)
        y = (d * rstd[:, None] * s["weight"] + s["bias"]).to(dt)
        return (y, mean, rstd) if c["save"] else y
    if c["from8"]:
        x = _held8(x)
    dy = s["dy"].float()
    xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"]
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if c["residual"]:
        dx = dx + s["dres"].float()
    return dx.to(dt), (dy * xh).sum(0), dy.sum(0)


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_held8(v):
    out = torch.empty_like(v)
    k = v.shape[1]
    whole = k // GROUP * GROUP
    for lo, hi, width in ((0, whole, GROUP), (whole, k, k - whole)):
        if hi == lo:
            continue
        part = v[:, lo:hi].reshape(v.shape[0], -1, width)
        frac, e = torch.frexp(part.abs().amax(-1, keepdim=True))
        e = e - 7 + (frac * 128.0 >= 127.5).to(e.dtype)
        e = e.clamp(-126, 121).double()
        step = torch.exp2(e)
        out[:, lo:hi] = (torch.round(part / step).clamp(-127, 127) * step).reshape(v.shape[0], -1)
    return out


def _exact_act(z, act):
    """act(z) and its slope."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        on = z > 0
        return torch.where(on, z, torch.zeros_like(z)), on.double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
    return z * cdf, cdf + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    x = s["x"].double()
    if op == "checkpoint":
        return _exact_held8(x)
    if op == "layer_norm":
        k = x.shape[1]
        mean = x.sum(1) / k
        x -= mean[:, None]
        rstd = torch.pow((x * x).sum(1) / k + EPS, -0.5)
        y = x.mul_(rstd[:, None]).mul_(s["weight"].double()).add_(s["bias"].double())
        return (y, mean, rstd) if case["save"] else y
    dy = s["dy"].double() if "dy" in s else None
    if op == "layer_norm_backward":
        k = x.shape[1]
        rstd = s["rstd"].double()[:, None]
        xh = ((_exact_held8(x) if case["from8"] else x) - s["mean"].double()[:, None]) * rstd
        dyw = dy * s["weight"].double()
        dx = rstd / k * (k * dyw - dyw.sum(1, keepdim=True) - xh * (dyw * xh).sum(1, keepdim=True))
        if case["residual"]:
            dx += s["dres"].double()
        return dx, (dy * xh).sum(0), dy.sum(0)
    w = s["w"].double()
    if op == "linear_backward":
        if "z" in s:
            dy = dy * _exact_act(s["z"].double(), case["act"])[1]
        return torch.matmul(dy, w), torch.matmul(dy.t(), x), dy.sum(0)
    z = torch.nn.functional.linear(x, w, s["bias"].double())
    y = _exact_act(z, case["act"])[0]
    if op == "linear_step8":
        dz = dy * _exact_act(_exact_held8(z), case["act"])[1]
        return y, torch.matmul(dz, w), torch.matmul(dz.t(), _exact_held8(x)), dz.sum(0)
    if case["residual"]:
        y = y + s["residual"].double()
    return (y, z) if case["save"] == "z" else y


def work(case):
    op, m, k = case["op"], case["m"], case["k"]
    e = 4 if case["dtype"] == "f32" else 2
    if op.startswith("linear"):
        n = case["n"]
        # forward: x, w, bias and the residual read, y (and z) written
        fwd = e * (m * k + n * k + m * n * (1 + case["residual"] + (case["save"] == "z"))) + 4 * n
        # backward: dy, x, w (and z) read, dx, dw and dbias written
        bwd = e * (m * n * (1 + (case["act"] != "none")) + 2 * m * k + 2 * n * k) + 4 * n
        flops = 2.0 * m * k * n
        if op == "linear":
            return {"bytes": fwd, "flops": flops}
        if op == "linear_backward":
            return {"bytes": bwd, "flops": 2 * flops}
        # the checkpoints: one byte a value and one a group of 32, written and read, in the place of z and x
        held = m * (k + -(-k // GROUP)) + (m * (n + -(-n // GROUP)) if case["act"] != "none" else 0)
        saved = e * (m * k + (m * n if case["act"] != "none" else 0))
        return {"bytes": fwd + bwd - saved + 2 * held, "flops": 3 * flops}
    if op == "layer_norm":
        return {"bytes": 2 * e * m * k + 8 * k + (8 * m if case["save"] else 0), "flops": 8.0 * m * k}
    if op == "layer_norm_backward":
        b = e * m * k * (3 + case["residual"]) + 8 * m + 12 * k
        if case["from8"]:
            b += 2 * m * (k + -(-k // GROUP))
        return {"bytes": b, "flops": 14.0 * m * k}
    return {"bytes": 2 * e * m * k + 2 * m * (k + -(-k // GROUP)), "flops": 6.0 * m * k}
