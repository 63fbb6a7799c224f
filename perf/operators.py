"""The operators of a channels-last block around the oriented convolution, as a user calls them: layer norm and its
gradients, the matrix product with bias, activation and residual in its epilogue and its gradients, and activation
checkpoints in 8 bits with their use in the backward pass.

Rows are pixels (or tokens), M of them; columns are features.  `pad` > 0: the input is a slice of a tensor that is
`pad` columns wider.  An 8-bit checkpoint holds groups of 64 columns of a row as integers in [-127, 127] and one float32 scale;
the integers' rows are padded to 16 bytes.
"""
import math

import torch

own = False

GROUP = 64
EPS = 1e-6
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # Layer norm after the convolution, first stage of a 64-image batch at 56 x 56: the largest, bound by memory.
        {"name": "ln_fwd 200704x96 bf16", "op": "ln_fwd", "M": 200704, "C": 96, "dt": "bf16", "pad": 0},
        # One image's last stage (7 x 7) in float32: a small call, where latency counts.
        {"name": "ln_fwd 49x768 f32", "op": "ln_fwd", "M": 49, "C": 768, "dt": "f32", "pad": 0},
        # Its backward at the second stage, 64 x 28 x 28, in float32.
        {"name": "ln_bwd 50176x192 f32", "op": "ln_bwd", "M": 50176, "C": 192, "dt": "f32", "packed": False},
        # The backward from an 8-bit checkpoint of the input, odd rows and columns (pruned widths).
        {"name": "ln_bwd 33333x211 bf16 packed", "op": "ln_bwd", "M": 33333, "C": 211, "dt": "bf16", "packed": True},
        # The block's first product, third stage of 64 images (14 x 14), with GELU, the pre-activation kept in 8 bits and used
        # for the gradient through the second product: the training step of the hidden layer.
        {"name": "step 12544 384-1536-384 bf16", "op": "step", "M": 12544, "I": 384, "O": 1536, "dt": "bf16",
         "act": "gelu"},
        # The block's second product with its residual, second stage, float32.
        {"name": "linear 50176 768-192 f32 res", "op": "linear", "M": 50176, "I": 768, "O": 192, "dt": "f32",
         "act": "none", "bias": True, "res": True, "save": False, "pad": 0},
        # A classifier's product for a batch of 16: few rows, bound by the weights and by latency.
        {"name": "linear 16 768-1000 bf16", "op": "linear", "M": 16, "I": 768, "O": 1000, "dt": "bf16",
         "act": "none", "bias": True, "res": False, "save": False, "pad": 0},
        # Odd widths and a slice as input, the pre-activation kept whole.
        {"name": "linear 9409 203-509 bf16 silu", "op": "linear", "M": 9409, "I": 203, "O": 509, "dt": "bf16",
         "act": "silu", "bias": True, "res": True, "save": True, "pad": 5},
        # The input gradient of the second product in float32 with the activation's derivative, third stage of 16 images.
        {"name": "bwd_input 3136 384-1536 f32", "op": "bwd_input", "M": 3136, "I": 1536, "O": 384, "dt": "f32",
         "act": "gelu", "packed": False},
        # Weight gradient of the second product from the 8-bit checkpoint of its input's pre-activation, second stage.
        {"name": "bwd_weight 50176 768-192 bf16", "op": "bwd_weight", "M": 50176, "I": 768, "O": 192, "dt": "bf16",
         "act": "gelu", "packed": True},
        # Weight gradient of the first product, first stage, float32: the longest sum.
        {"name": "bwd_weight 200704 96-384 f32", "op": "bwd_weight", "M": 200704, "I": 96, "O": 384, "dt": "f32",
         "act": "none", "packed": False},
        # A checkpoint written and read back: the hidden layer of the second stage.
        {"name": "ckpt 50176x768 bf16", "op": "ckpt", "M": 50176, "C": 768, "dt": "bf16"},
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; half of them odd, the others whole eights where they are large enough."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        n |= 1
    elif n >= 16:
        n -= n % 8
    n = max(lo, min(hi, n))
    return n if n != 3072 else 3071


def draw(rng):
    most_b = max(work(c)["bytes"] for c in listed())
    most_f = max(work(c)["flops"] for c in listed())
    while True:
        op = rng.choice(["ln_fwd", "ln_bwd", "linear", "linear", "bwd_input", "bwd_weight", "step", "ckpt"])
        dt = rng.choice(["f32", "bf16"])
        c = {"op": op, "M": _size(rng, 1, 200704), "dt": dt}
        if op in ("ln_fwd", "ln_bwd", "ckpt"):
            c["C"] = _size(rng, 1, 2048)
        else:
            c["I"], c["O"] = _size(rng, 8, 2048), _size(rng, 8, 2048)
        act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
        if op == "ln_fwd":
            c["pad"] = rng.choice([0, 0, 8, 13])
        elif op == "ln_bwd":
            c["packed"] = rng.random() < 0.5
        elif op == "linear":
            c.update(act=act, bias=rng.random() < 0.75, res=rng.random() < 0.5, save=rng.random() < 0.5,
                     pad=rng.choice([0, 0, 8, 13]))
        elif op in ("bwd_input", "bwd_weight"):
            c.update(act=act, packed=rng.random() < 0.5)
        elif op == "step":
            # (bfloat16: where float32 values round to 8 bits, the last bit of a product decides a whole step)
            c.update(act=act if act != "none" else "gelu", dt="bf16")
        w = work(c)
        if w["bytes"] <= most_b and w["flops"] <= most_f:
            return c


def work(c):
    M, es, op = c["M"], 4 if c["dt"] == "f32" else 2, c["op"]

    def held(cols):  # an 8-bit checkpoint
        return M * (cols + 4 * -(-cols // GROUP))

    if op == "ln_fwd":
        return {"bytes": 2 * M * c["C"] * es + 2 * c["C"] * es + 8 * M, "flops": 8 * M * c["C"]}
    if op == "ln_bwd":
        x = held(c["C"]) if c["packed"] else M * c["C"] * es
        return {"bytes": 2 * M * c["C"] * es + x + 8 * M + 3 * c["C"] * es, "flops": 14 * M * c["C"]}
    if op == "ckpt":
        return {"bytes": 2 * M * c["C"] * es + 2 * held(c["C"]), "flops": 4 * M * c["C"]}
    I, O = c["I"], c["O"]
    if op == "linear":
        outs = 1 + c["res"] + c["save"]
        return {"bytes": es * (M * I + I * O + O * c["bias"] + outs * M * O), "flops": 2 * M * I * O}
    if op == "bwd_input":
        pre = 0 if c["act"] == "none" else (held(I) if c["packed"] else M * I * es)
        return {"bytes": es * (M * O + I * O + M * I) + pre, "flops": 2 * M * I * O}
    if op == "bwd_weight":
        x = held(I) if c["packed"] else M * I * es
        return {"bytes": es * (M * O + I * O + O) + x, "flops": 2 * M * I * O}
    # step: the product with its activation, its checkpoint written and read, the product's gradient through it
    return {"bytes": es * (2 * M * I + 2 * I * O + O + 2 * M * O) + 2 * held(O), "flops": 4 * M * I * O}


# ---------------------------------------------------------------- inputs

def _hold(x):
    """The 8-bit checkpoint of a float32 tensor in its plain form: integers (rows padded to 16) and scales."""
    M, C = x.shape
    groups = -(-C // GROUP)
    g = torch.nn.functional.pad(x, (0, groups * GROUP - C)).view(M, groups, GROUP)
    amax = g.abs().amax(-1)
    fine = torch.isfinite(g).all(-1)
    some = fine & (amax >= 2.0 ** -100)
    inv = torch.where(some, torch.full_like(amax, 127.0) / amax, torch.zeros_like(amax))
    q = torch.where(some[..., None], torch.round(g * inv[..., None]), torch.zeros_like(g)).to(torch.int8)
    scale = torch.where(some, amax / 127.0, torch.where(fine, torch.zeros_like(amax), torch.full_like(amax, math.nan)))
    held = torch.zeros(M, -(-C // 16) * 16, dtype=torch.int8, device=x.device)
    held[:, :C] = q.view(M, groups * GROUP)[:, :C]
    return held, scale.contiguous()


def _stands_for(held, scale, C):
    return held[:, :C].float() * scale.repeat_interleave(GROUP, 1)[:, :C]


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, M, op = _DT[c["dt"]], c["M"], c["op"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    def rows(cols, pad=0):
        # features have their own sizes and offsets, as a convolution's outputs have
        size = torch.rand(cols + pad, generator=gen, device="cuda") + 0.5
        x = (normal(M, cols + pad) * size + normal(cols + pad, std=0.5)).to(dt)
        return x[:, :cols]

    s = {"case": dict(c)}
    if op in ("ln_fwd", "ln_bwd"):
        C = c["C"]
        s["w"], s["b"] = (1 + normal(C, std=0.1)).to(dt), normal(C, std=0.1).to(dt)
        x = rows(C, c.get("pad", 0))
        if op == "ln_bwd":
            f = x.float()
            s["mean"] = f.mean(1)
            s["rstd"] = (f.var(1, unbiased=False) + EPS).rsqrt()
            s["dy"] = normal(M, C).to(dt)
            if c["packed"]:
                s["held"], s["scale"] = _hold(f)
                return s
        s["x"] = x
    elif op == "ckpt":
        s["x"] = rows(c["C"])
    else:
        I, O = c["I"], c["O"]
        s["w"] = normal(O, I, std=I ** -0.5).to(dt)
        if op in ("linear", "step"):
            s["x"] = rows(I, c.get("pad", 0))
            s["b"] = normal(O, std=0.1).to(dt) if c.get("bias", True) else None
            if c.get("res"):
                s["res"] = normal(M, O).to(dt)
            if op == "step":
                s["w2"] = normal(I, O, std=O ** -0.5).to(dt)
                s["dy"] = normal(M, I).to(dt)
        else:
            s["dy"] = normal(M, O).to(dt)
            x = rows(I)  # the pre-activation of the product's input
            if op == "bwd_weight":
                del s["w"]
            if c["packed"]:
                s["held"], s["scale"] = _hold(x.float())
            else:
                s["x"] = x.contiguous()
    return s


# ---------------------------------------------------------------- one pass

def _act(h, act):
    if act == "relu":
        return torch.where(h > 0, h, torch.zeros_like(h))
    if act == "gelu":
        return 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * h * (1 + torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h * h * h)))
    if act == "silu":
        return h * torch.sigmoid(h)
    return h


def _slope(h, act):
    if act == "relu":
        return (h > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(h * math.sqrt(0.5))) + h * torch.exp(-0.5 * h * h) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        r = math.sqrt(2 / math.pi)
        t = torch.tanh(r * (h + 0.044715 * h * h * h))
        return 0.5 * (1 + t) + 0.5 * h * (1 - t * t) * r * (1 + 3 * 0.044715 * h * h)
    if act == "silu":
        g = torch.sigmoid(h)
        return g * (1 + h * (1 - g))
    return torch.ones_like(h)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    c = s["case"]
    op, dt = c["op"], _DT[c["dt"]]
    if op == "ln_fwd":
        x = s["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = ((d * d).mean(1) + EPS).rsqrt()
        return (d * rstd[:, None] * s["w"].float() + s["b"].float()).to(dt), mean, rstd
    if op == "ln_bwd":
        x = _stands_for(s["held"], s["scale"], c["C"]) if c["packed"] else s["x"].float()
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = (x - s["mean"][:, None]) * rstd
        g = dy * s["w"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return dx.to(dt), (dy * xh).sum(0).to(dt), dy.sum(0).to(dt)
    if op == "ckpt":
        return _stands_for(*_hold(s["x"].float()), c["C"]).to(dt)
    if op == "linear":
        h = s["x"].float() @ s["w"].float().t()
        if c["bias"]:
            h = h + s["b"].float()
        y = _act(h, c["act"])
        if c["res"]:
            y = y + s["res"].float()
        return (y.to(dt), h.to(dt)) if c["save"] else y.to(dt)
    if op == "step":
        h = s["x"].float() @ s["w"].float().t() + s["b"].float()
        pre = _stands_for(*_hold(h), c["O"])
        dh = (s["dy"].float() @ s["w2"].float()) * _slope(pre, c["act"])
        return _act(h, c["act"]).to(dt), dh.to(dt)
    x = _stands_for(s["held"], s["scale"], c["I"]) if c["packed"] else s["x"].float()
    dy = s["dy"].float()
    if op == "bwd_input":
        return ((dy @ s["w"].float()) * _slope(x, c["act"])).to(dt)
    return (dy.t() @ _act(x, c["act"])).to(dt), dy.sum(0).to(dt)


def _run_own(s):
    from paper_2309_15812_amd import ops

    c = s["case"]
    op = c["op"]
    if op == "ln_fwd":
        return ops.ln_fwd(s["x"], s["w"], s["b"], eps=EPS)
    if op == "ckpt":
        return ops.unpack8(ops.pack8(s["x"]), _DT[c["dt"]])
    if op == "linear":
        return ops.linear_fwd(s["x"], s["w"], s["b"], act=c["act"], residual=s.get("res"),
                              save="pre" if c["save"] else None)
    if op == "step":
        y, held = ops.linear_fwd(s["x"], s["w"], s["b"], act=c["act"], save="pack8")
        return y, ops.linear_bwd_input(s["dy"], s["w2"], pre=held, act=c["act"])
    x = ops.Packed8(s["held"], s["scale"], c["C"] if op == "ln_bwd" else c["I"]) if c["packed"] else s["x"]
    if op == "ln_bwd":
        return ops.ln_bwd(x, s["dy"], s["mean"], s["rstd"], s["w"])
    if op == "bwd_input":
        return ops.linear_bwd_input(s["dy"], s["w"], pre=x if c["act"] != "none" else None, act=c["act"])
    return ops.linear_bwd_weight(x, s["dy"], act=c["act"])


# ---------------------------------------------------------------- the definition in 64 bits

def _gate64(h, act):
    """(value, derivative) of an activation in 64 bits."""
    if act == "none":
        return h, torch.ones_like(h)
    if act == "relu":
        return h.clamp(min=0), (h > 0).double()
    if act == "silu":
        g = 1 / (1 + torch.exp(-h))
        return h * g, g + h * g * (1 - g)
    if act == "gelu":
        area = 0.5 * torch.special.erfc(-h / math.sqrt(2.0))
        return h * area, area + h * torch.exp(-h * h / 2) / math.sqrt(2 * math.pi)
    k = 2 * math.sqrt(2 / math.pi)  # (1 + tanh u) / 2 is the logistic function of 2 u
    g = 1 / (1 + torch.exp(-k * (h + 0.044715 * h ** 3)))
    return h * g, g + h * g * (1 - g) * k * (1 + 0.134145 * h * h)


def _held64(x):
    """What an 8-bit checkpoint of x stands for, in 64 bits."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[1], GROUP):
        g = x[:, at:at + GROUP]
        step = g.abs().max(1, keepdim=True).values / 127
        out[:, at:at + GROUP] = torch.where(step > 0, torch.round(g / step.clamp(min=1e-300)) * step, g * 0)
    return out


def exact(c, seed):
    s = prepare(c, seed)
    op = c["op"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if op != "ckpt" and "held" in d:
        cols = c["C"] if op == "ln_bwd" else c["I"]
        at = torch.arange(cols, device="cuda") // GROUP
        d["x"] = d["held"][:, :cols] * d["scale"][:, at]
    if op == "ln_fwd":
        var, mean = torch.var_mean(d["x"], 1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        return (d["x"] - mean[:, None]) * rstd[:, None] * d["w"] + d["b"], mean, rstd
    if op == "ln_bwd":
        C = c["C"]
        xh = (d["x"] - d["mean"][:, None]) * d["rstd"][:, None]
        g = d["dy"] * d["w"]
        sums = torch.stack((g.sum(1), (g * xh).sum(1)))
        dx = (C * g - sums[0][:, None] - xh * sums[1][:, None]) * (d["rstd"][:, None] / C)
        return dx, torch.einsum("mc,mc->c", d["dy"], xh), torch.ones(c["M"], device="cuda").double() @ d["dy"]
    if op == "ckpt":
        return _held64(d["x"])
    if op in ("linear", "step"):
        h = torch.mm(d["w"], d["x"].t()).t().contiguous()
        if "b" in d:
            h += d["b"]
        y = _gate64(h, c["act"])[0]
        if op == "linear":
            if "res" in d:
                y = y + d["res"]
            return (y, h) if c["save"] else y
        return y, torch.mm(d["w2"].t(), d["dy"].t()).t() * _gate64(_held64(h), c["act"])[1]
    if op == "bwd_input":
        return torch.mm(d["w"].t(), d["dy"].t()).t() * _gate64(d["x"], c["act"])[1]
    return torch.mm(_gate64(d["x"], c["act"])[0].t(), d["dy"]).t(), torch.ones(c["M"], device="cuda").double() @ d["dy"]
