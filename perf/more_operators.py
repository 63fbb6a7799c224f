"""Operators of a training step around the oriented convolution, as a user calls them: group norm with an activation on
channels-last activations and its gradients, matrix products of 8-bit floating point operands with a scale for each 128 values of
a row, and an AdamW step over all tensors of a model.

Group norm: x is (N, P, C), P pixels of a sample, C = G D channels in G groups; a group's statistics are those of its P D values.

8-bit operands: a matrix of R rows of K values is held as e4m3 or e5m2 (R, K rounded up to 128; zeros behind the row's end) and
exponents (ceil(K / 128), R rounded up to 16; 127 behind the last row).  Value k of row r stands for q[r, k] 2^(e[k / 128, r] - 127).
The power of two is the least one that keeps the group's finite values in the type's range; zeros have e = 127 and a value
that is not finite becomes NaN.  A product reads two such operands along the same axis, so a matrix that is read along both
is held twice, by rows and transposed.

AdamW: the states of all tensors are flat, each tensor's part starts at a multiple of 128.  In 8 bits, m and the root of v
are e4m3 with one float32 scale for each 128 values; a positive root is at least the type's smallest value.  With max_norm,
the gradients are scaled down to that norm over all tensors, and nothing is changed where the norm is not finite.
"""
import math

import torch

own = False

EPS = 1e-5
GROUP = 128
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_TOP = {"e4m3": 448.0, "e5m2": 57344.0}
LR, BETAS, ADAM_EPS, DECAY = 1e-3, (0.9, 0.999), 1e-8, 0.05


def listed():
    return [
        # The norm after the convolution at the first stage of a 64-image batch at 56 x 56: memory, 3 channels a group.
        {"name": "gn_fwd 64x3136x96 g32 bf16", "op": "gn_fwd", "N": 64, "P": 3136, "G": 32, "D": 3, "dt": "bf16",
         "act": "silu"},
        # One image's last stage (7 x 7) in float32: a small call, where latency counts.
        {"name": "gn_fwd 1x49x768 g32 f32", "op": "gn_fwd", "N": 1, "P": 49, "G": 32, "D": 24, "dt": "f32", "act": "gelu"},
        # The gradients at the second stage, 64 x 28 x 28, in float32.
        {"name": "gn_bwd 64x784x192 g32 f32", "op": "gn_bwd", "N": 64, "P": 784, "G": 32, "D": 6, "dt": "f32", "act": "silu"},
        # Few large odd images (97 x 131 crops) and a pruned width.
        {"name": "gn_bwd 3x12707x203 g7 bf16", "op": "gn_bwd", "N": 3, "P": 12707, "G": 7, "D": 29, "dt": "bf16",
         "act": "gelu"},
        # The hidden layer's first product in training, third stage of 64 images, the pre-activation kept.
        {"name": "f8_fwd 12544 384-1536 bf16", "op": "f8_fwd", "M": 12544, "I": 384, "O": 1536, "dt": "bf16", "act": "gelu",
         "bias": True, "res": False, "save": True, "fmt": "e4m3"},
        # A large square product: the matrix cores' rate.
        {"name": "f8_fwd 8192 8192-8192 bf16", "op": "f8_fwd", "M": 8192, "I": 8192, "O": 8192, "dt": "bf16", "act": "none",
         "bias": False, "res": False, "save": False, "fmt": "e4m3"},
        # A classifier's product for a batch of 16: the weights and latency.
        {"name": "f8_fwd 16 768-1000 f32", "op": "f8_fwd", "M": 16, "I": 768, "O": 1000, "dt": "f32", "act": "none",
         "bias": True, "res": False, "save": False, "fmt": "e4m3"},
        # The gradient through the second product and the activation before it, third stage; gradients in e5m2.
        {"name": "f8_bwd_input 12544 384-1536", "op": "f8_bwd_input", "M": 12544, "I": 1536, "O": 384, "dt": "bf16",
         "act": "gelu", "fmt": "e5m2"},
        # The weight gradient of the second product, second stage: a long sum; the input is kept in 8 bits.
        {"name": "f8_bwd_weight 50176 768-192", "op": "f8_bwd_weight", "M": 50176, "I": 768, "O": 192, "dt": "bf16",
         "fmt": "e4m3"},
        # The tensors of three stages of blocks (7 tensors each) in float32 with 32-bit states, their gradients' norm limited.
        {"name": "adamw 96x3 192x3 384x9 f32", "op": "adamw", "dims": "96x3 192x3 384x9", "K": 31, "dt": "f32", "gdt": "f32",
         "bits": 32, "master": False, "clip": True},
        # The same tensors in bfloat16 with their float32 values and 8-bit states.
        {"name": "adamw 96x3 192x3 384x9 bf16 8", "op": "adamw", "dims": "96x3 192x3 384x9", "K": 31, "dt": "bf16",
         "gdt": "bf16", "bits": 8, "master": True, "clip": False},
        # One small block of an odd width: launches.
        {"name": "adamw 33x1 f32 8", "op": "adamw", "dims": "33x1", "K": 7, "dt": "f32", "gdt": "f32", "bits": 8,
         "master": False, "clip": True},
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; half of them odd, the others whole eights where they are large enough."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        n |= 1
    elif n >= 16:
        n -= n % 8
    return max(lo, min(hi, n))


def draw(rng):
    cost = {}
    for c in listed():
        kind, w = c["op"][:2], work(c)
        cost[kind] = [max(a, b) for a, b in zip(cost.get(kind, (0, 0)), (w["bytes"], w["flops"]))]
    while True:
        op = rng.choice(["gn_fwd", "gn_bwd", "f8_fwd", "f8_fwd", "f8_bwd_input", "f8_bwd_weight", "adamw", "adamw"])
        dt = rng.choice(["f32", "bf16"])
        act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
        if op.startswith("gn"):
            # (a group of few values has a gradient that is all cancellation)
            c = {"op": op, "N": _size(rng, 1, 256), "P": _size(rng, 1, 50176), "G": _size(rng, 1, 64), "D": _size(rng, 1, 64),
                 "dt": dt, "act": act}
            if c["P"] * c["D"] < 16:
                continue
        elif op.startswith("f8"):
            c = {"op": op, "M": _size(rng, 1, 100352), "I": _size(rng, 8, 8192), "O": _size(rng, 8, 8192), "dt": dt,
                 "fmt": rng.choice(["e4m3", "e5m2"])}
            if op != "f8_bwd_weight":
                c["act"] = act
            if op == "f8_fwd":
                c.update(fmt="e4m3", bias=rng.random() < 0.75, res=rng.random() < 0.5, save=rng.random() < 0.5)
        else:
            dims = " ".join("%dx%d" % (_size(rng, 8, 512), rng.randint(1, 6)) for _ in range(rng.randint(1, 4)))
            c = {"op": op, "dims": dims, "K": rng.choice([3, 7, 15, 31]), "dt": dt, "gdt": dt, "bits": rng.choice([8, 32]),
                 "master": dt == "bf16" and rng.random() < 0.7, "clip": rng.random() < 0.5}
        w = work(c)
        if w["bytes"] <= cost[op[:2]][0] and w["flops"] <= cost[op[:2]][1]:
            return c


def _shapes(c):
    """The tensors of residual blocks of the widths and depths in c["dims"], hidden layers four times as wide."""
    got = []
    for part in c["dims"].split():
        C, depth = map(int, part.split("x"))
        got += [(C, c["K"]), (C,), (C,), (4 * C, C), (4 * C,), (C, 4 * C), (C,)] * depth
    return got


def work(c):
    op, es = c["op"], 4 if c["dt"] == "f32" else 2
    if op.startswith("gn"):
        n, C = c["N"] * c["P"] * c["G"] * c["D"], c["G"] * c["D"]
        stats = 8 * c["N"] * c["G"]
        if op == "gn_fwd":
            return {"bytes": 2 * n * es + 2 * C * es + stats, "flops": 10 * n}
        return {"bytes": 3 * n * es + 4 * C * es + stats, "flops": 25 * n}
    if op == "adamw":
        n = sum(math.prod(s) for s in _shapes(c))
        state = 16 if c["bits"] == 32 else 4 + 16 / GROUP
        return {"bytes": n * (2 * es + (4 if c["gdt"] == "f32" else 2) + state + 8 * c["master"]), "flops": 15 * n}
    M, I, O = c["M"], c["I"], c["O"]

    def held(rows, cols):
        return rows * (cols + -(-cols // GROUP))

    if op == "f8_fwd":
        outs = 1 + c["res"] + c["save"]
        return {"bytes": es * (M * I + O * c["bias"] + outs * M * O) + held(O, I), "flops": 2 * M * I * O}
    if op == "f8_bwd_input":
        return {"bytes": es * (M * O + M * I * (1 + (c["act"] != "none"))) + held(I, O), "flops": 2 * M * I * O}
    return {"bytes": es * (M * O + I * O + O) + held(I, M), "flops": 2 * M * I * O}


# ---------------------------------------------------------------- inputs

def _pack(x, fmt):
    """(q, e) of a float32 matrix in the plain form."""
    R, K = x.shape
    groups = -(-K // GROUP)
    g = torch.nn.functional.pad(x, (0, groups * GROUP - K)).view(R, groups, GROUP)
    fine = torch.isfinite(g)
    amax = torch.where(fine, g, torch.zeros_like(g)).abs().amax(-1)
    m, p = torch.frexp(amax)  # amax = m 2^p, 0.5 <= m < 1; the types' largest values are 0.875 of a power of two
    e = (p - (9 if fmt == "e4m3" else 16) + (m > 0.875).to(p.dtype)).clamp(-127, 127)
    e = torch.where(amax > 0, e, torch.zeros_like(e))
    q = torch.where(fine, g * torch.exp2(-e.float())[..., None], torch.full_like(g, math.nan)).to(_F8[fmt])
    exponents = torch.full((groups, -(-R // 16) * 16), 127, dtype=torch.uint8, device=x.device)
    exponents[:, :R] = (e + 127).to(torch.uint8).t()
    return q.view(R, groups * GROUP), exponents


def _stands_for(q, e, K):
    R = q.shape[0]
    scale = torch.exp2(e[:, :R].float() - 127).t()
    return (q.float().view(R, -1, GROUP) * scale[..., None]).view(R, -1)[:, :K]


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, op = _DT[c["dt"]], c["op"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    def features(*shape):
        # features have their own sizes and offsets, as a convolution's outputs have
        size = torch.rand(shape[-1], generator=gen, device="cuda") + 0.5
        return (normal(*shape) * size + normal(shape[-1], std=0.5)).to(dt)

    s = {"case": dict(c)}
    if op.startswith("gn"):
        N, P, G, C = c["N"], c["P"], c["G"], c["G"] * c["D"]
        s["w"], s["b"] = (1 + normal(C, std=0.1)).to(dt), normal(C, std=0.1).to(dt)
        s["x"] = features(N, P, C)
        if op == "gn_bwd":
            v = s["x"].double().view(N, P, G, c["D"])
            s["mean"] = v.mean((1, 3)).float()
            s["rstd"] = (v.var((1, 3), unbiased=False) + EPS).rsqrt().float()
            s["dy"] = normal(N, P, C).to(dt)
    elif op == "adamw":
        shapes = _shapes(c)
        total = sum(math.prod(t) for t in shapes)
        starts, padded = [], 0
        for t in shapes:
            starts.append(padded)
            padded += -(-math.prod(t) // GROUP) * GROUP
        # parameters and gradients lie one behind the other, as in a program that keeps them in one buffer
        s["flat_p"], s["flat_g"] = normal(total, std=0.05).to(dt), normal(total, std=0.02).to(_DT[c["gdt"]])
        sizes = [math.prod(t) for t in shapes]
        s["p"] = [t.view(shape) for t, shape in zip(s["flat_p"].split(sizes), shapes)]
        s["g"] = [t.view(shape) for t, shape in zip(s["flat_g"].split(sizes), shapes)]
        s["sizes"], s["starts"] = sizes, starts
        # a state after some steps: m near the gradients, v near their squares, tensors of different sizes of gradients
        inside = torch.zeros(padded, dtype=torch.bool, device="cuda")
        size = torch.empty(padded, device="cuda")
        for n, at in zip(sizes, starts):
            inside[at:at + n] = True
            size[at:at + n] = math.exp(float(torch.randn((), generator=gen, device="cuda")))
        m = torch.where(inside, normal(padded, std=0.01) * size, torch.zeros_like(size))
        r = torch.where(inside, (torch.rand(padded, generator=gen, device="cuda") + 0.2) * 0.03 * size, torch.zeros_like(size))
        if c["master"]:
            s["master"] = torch.zeros(padded, device="cuda")
            for p, n, at in zip(s["p"], sizes, starts):
                s["master"][at:at + n] = p.reshape(-1).float() * (1 + normal(n, std=1e-3))
        if c["bits"] == 8:
            s["m"], s["ms"] = _to8(m)
            s["v"], s["vs"] = _to8(r, least=True)
        else:
            s["m"], s["v"] = m, r * r
        s["step"] = torch.tensor([20, 0], dtype=torch.int32, device="cuda")
    else:
        M, I, O = c["M"], c["I"], c["O"]
        if op == "f8_fwd":
            s["x"] = features(M, I)
            s["wq"], s["we"] = _pack(normal(O, I, std=I ** -0.5), "e4m3")
            s["b"] = normal(O, std=0.1).to(dt) if c["bias"] else None
            s["res"] = normal(M, O).to(dt) if c["res"] else None
        elif op == "f8_bwd_input":
            s["dy"] = normal(M, O).to(dt)
            s["wq"], s["we"] = _pack(normal(I, O, std=O ** -0.5), "e4m3")  # the weights transposed
            s["pre"] = features(M, I) if c["act"] != "none" else None
        else:
            s["dy"] = normal(M, O).to(dt)
            s["xq"], s["xe"] = _pack(features(M, I).float().t().contiguous(), "e4m3")  # the product's input transposed
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


def _to8(t, least=False):
    """(e4m3 values, scales) of a flat state whose length is a multiple of 128."""
    g = t.view(-1, GROUP)
    amax = g.abs().amax(1)
    some = amax > 0
    inv = torch.where(some, 448.0 / amax, torch.zeros_like(amax))
    u = g * inv[:, None]
    if least:
        u = torch.where(g > 0, u.clamp(min=2.0 ** -9), u)
    return u.to(torch.float8_e4m3fn).view(-1), amax / 448.0


def _from8(q, scale):
    return (q.float().view(-1, GROUP) * scale[:, None]).view(-1)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    c = s["case"]
    op, dt = c["op"], _DT[c["dt"]]
    if op == "gn_fwd":
        N, P, G, D = c["N"], c["P"], c["G"], c["D"]
        x = s["x"].float().view(N, P, G, D)
        mean = x.mean((1, 3))
        d = x - mean[:, None, :, None]
        rstd = ((d * d).mean((1, 3)) + EPS).rsqrt()
        h = (d * rstd[:, None, :, None]).view(N, P, G * D) * s["w"].float() + s["b"].float()
        return _act(h, c["act"]).to(dt), mean, rstd
    if op == "gn_bwd":
        N, P, G, D = c["N"], c["P"], c["G"], c["D"]
        rstd = s["rstd"][:, None, :, None]
        xh = (s["x"].float().view(N, P, G, D) - s["mean"][:, None, :, None]) * rstd
        flat = xh.view(N, P, G * D)
        dh = s["dy"].float() * _slope(flat * s["w"].float() + s["b"].float(), c["act"])
        g = (dh * s["w"].float()).view(N, P, G, D)
        dx = rstd * (g - g.mean((1, 3), keepdim=True) - xh * (g * xh).mean((1, 3), keepdim=True))
        return dx.view(N, P, G * D).to(dt), (dh * flat).sum((0, 1)).to(dt), dh.sum((0, 1)).to(dt)
    if op == "adamw":
        return _adamw_plain(s)
    if op == "f8_fwd":
        x = _stands_for(*_pack(s["x"].float(), "e4m3"), c["I"])
        h = x @ _stands_for(s["wq"], s["we"], c["I"]).t()
        if c["bias"]:
            h = h + s["b"].float()
        y = _act(h, c["act"])
        if c["res"]:
            y = y + s["res"].float()
        return (y.to(dt), h.to(dt)) if c["save"] else y.to(dt)
    if op == "f8_bwd_input":
        dy = _stands_for(*_pack(s["dy"].float(), c["fmt"]), c["O"])
        dx = dy @ _stands_for(s["wq"], s["we"], c["O"]).t()
        return (dx if s["pre"] is None else dx * _slope(s["pre"].float(), c["act"])).to(dt)
    dy = s["dy"].float()
    q, e = _pack(dy.t().contiguous(), c["fmt"])
    dw = _stands_for(q, e, c["M"]) @ _stands_for(s["xq"], s["xe"], c["M"]).t()
    return dw.to(dt), dy.sum(0).to(dt)


def _adamw_plain(s):
    c = s["case"]
    step, (b1, b2) = s["step"], BETAS
    factor, ok, norm = None, None, None
    if c["clip"]:
        norm = s["flat_g"].double().square().sum().sqrt().float()
        ok = torch.isfinite(norm)
        factor = torch.where(norm > 1.0, 1.0 / norm, torch.ones_like(norm))
    t = (step[0] + 1).double()
    c1, c2 = (1 / (1 - torch.pow(b1, t))).float(), (1 / (1 - torch.pow(b2, t))).sqrt().float()
    held8 = c["bits"] == 8
    m_all, v_all = s["m"], s["v"]
    if held8:
        m_all, r = _from8(m_all, s["ms"]), _from8(v_all, s["vs"])
        v_all = r * r
    new_m, new_v = torch.zeros_like(m_all), torch.zeros_like(v_all)
    # (a list of tensors, each with a part of the states)
    for p, g, n, at in zip(s["p"], s["g"], s["sizes"], s["starts"]):
        g = g.reshape(-1).float()
        if factor is not None:
            g = g * factor
        w = s["master"][at:at + n] if c["master"] else p.reshape(-1).float()
        m = b1 * m_all[at:at + n] + (1 - b1) * g
        v = b2 * v_all[at:at + n] + (1 - b2) * (g * g)
        new = w * (1 - LR * DECAY) - LR * ((m * c1) / (v.sqrt() * c2 + ADAM_EPS))
        new_m[at:at + n], new_v[at:at + n] = m, v
        if ok is not None:
            new = torch.where(ok, new, w)
        if c["master"]:
            s["master"][at:at + n] = new
        p.copy_(new.view(p.shape))
    held = [(new_m, None), (new_v, None)] if not held8 else [_to8(new_m), _to8(new_v.sqrt(), least=True)]
    for (value, scale), name in zip(held, "mv"):
        s[name].copy_(value if ok is None else torch.where(ok, value.float(), s[name].float()).to(value.dtype))
        if scale is not None:
            s[name + "s"].copy_(scale if ok is None else torch.where(ok, scale, s[name + "s"]))
    step[0] += 1 if ok is None else ok.to(step.dtype)
    return _adamw_outputs(s, norm)


def _adamw_outputs(s, norm):
    got = {k: s[k] for k in ("flat_p", "master", "m", "ms", "v", "vs", "step") if k in s}
    if norm is not None:
        got["norm"] = norm
    return got


def _run_own(s):
    from paper_2309_15812_amd import ops

    c = s["case"]
    op = c["op"]
    if op == "gn_fwd":
        return ops.gn_fwd(s["x"], s["w"], s["b"], c["G"], eps=EPS, act=c["act"])
    if op == "gn_bwd":
        return ops.gn_bwd(s["x"], s["dy"], s["mean"], s["rstd"], s["w"], s["b"], act=c["act"])
    if op == "adamw":
        state = ops.AdamState(s["sizes"], s["m"], s["v"], s["step"], s.get("ms"), s.get("vs"), s.get("master"))
        norm = ops.adamw(s["p"], s["g"], state, lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY,
                         max_norm=1.0 if c["clip"] else None)
        return _adamw_outputs(s, norm)
    dt = _DT[c["dt"]]
    if op == "f8_fwd":
        return ops.f8_linear_fwd(ops.pack_f8(s["x"]), ops.F8(s["wq"], s["we"], c["I"]), s["b"], act=c["act"],
                                 residual=s["res"], save="pre" if c["save"] else None, dtype=dt)
    if op == "f8_bwd_input":
        return ops.f8_linear_bwd_input(ops.pack_f8(s["dy"], c["fmt"]), ops.F8(s["wq"], s["we"], c["O"]), pre=s["pre"],
                                       act=c["act"], dtype=dt)
    dyt, db = ops.pack_f8(s["dy"], c["fmt"], along="rows", sums=True)
    return ops.f8_linear_bwd_weight(dyt, ops.F8(s["xq"], s["xe"], c["M"]), dtype=dt), db


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


def _nearest64(u, fmt):
    """u rounded to the type's values (ties to even), in 64 bits."""
    digits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    spacing = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** low))) - digits)
    return torch.round(u / spacing) * spacing


def _held64(x, fmt):
    """What an 8-bit operand made of x (groups along its last axis) stands for, in 64 bits."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[1], GROUP):
        g = x[:, at:at + GROUP]
        amax = g.abs().max(1, keepdim=True).values
        scale = torch.exp2(torch.ceil(torch.log2(amax.clamp(min=1e-300) / _TOP[fmt])))
        out[:, at:at + GROUP] = torch.where(amax > 0, _nearest64(g / scale, fmt) * scale, g * 0)
    return out


def _value64(q, e, K):
    scale = 2.0 ** (e[:, :q.shape[0]].double() - 127)
    return q[:, :K].double() * scale.t().repeat_interleave(GROUP, 1)[:, :K]


def _adam64(s):
    c = s["case"]
    inside = torch.cat([torch.arange(at, at + n, device="cuda") for n, at in zip(s["sizes"], s["starts"])])
    got = {k: s[k].double() for k in ("flat_p", "flat_g", "m", "v", "master", "ms", "vs") if k in s}
    m, v = got["m"], got["v"]
    if c["bits"] == 8:
        m = m * got["ms"].repeat_interleave(GROUP)
        v = (v * got["vs"].repeat_interleave(GROUP)) ** 2
    g = torch.zeros_like(m)
    g[inside] = got["flat_g"]
    norm = torch.linalg.vector_norm(g)
    if c["clip"]:
        g = g / max(1.0, float(norm))
    t = int(s["step"][0]) + 1
    w = torch.zeros_like(m)
    w[inside] = got["master"][inside] if c["master"] else got["flat_p"]
    m = m + (1 - BETAS[0]) * (g - m)
    v = v + (1 - BETAS[1]) * (g * g - v)
    rate = LR * math.sqrt(1 - BETAS[1] ** t) / (1 - BETAS[0] ** t)
    w = w - LR * DECAY * w - rate * m / (torch.sqrt(v) + ADAM_EPS * math.sqrt(1 - BETAS[1] ** t))
    out = {"flat_p": w[inside], "step": None}
    if c["master"]:
        out["master"] = w
    if c["clip"]:
        out["norm"] = norm
    if c["bits"] == 32:
        return out | {"m": m, "v": v}
    for name, value in (("m", m), ("v", torch.sqrt(v))):
        rows = value.view(-1, GROUP)
        top = rows.abs().max(1, keepdim=True).values / 448
        u = torch.where(top > 0, rows / top.clamp(min=1e-300), rows * 0)
        if name == "v":
            u = torch.where(rows > 0, u.clamp(min=2.0 ** -9), u)
        out[name], out[name + "s"] = _nearest64(u, "e4m3").view(-1), top[:, 0]
    return out


def exact(c, seed):
    s = prepare(c, seed)
    op = c["op"]
    if op == "adamw":
        return _adam64(s)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.dtype in _DT.values()}
    if op.startswith("gn"):
        N, P, G, D = c["N"], c["P"], c["G"], c["D"]
        x = d["x"].view(N, P, G, D).permute(0, 2, 1, 3).reshape(N, G, P * D)
        wb = [d[k].view(1, G, 1, D).expand(N, G, P, D).reshape(N, G, P * D) for k in "wb"]

        def back(v):
            return v.view(N, G, P, D).permute(0, 2, 1, 3).reshape(N, P, G * D)

        if op == "gn_fwd":
            var, mean = torch.var_mean(x, 2, correction=0)
            rstd = 1 / torch.sqrt(var + EPS)
            h = (x - mean[..., None]) * rstd[..., None] * wb[0] + wb[1]
            return back(_gate64(h, c["act"])[0]), mean, rstd
        n = P * D
        xh = (x - d["mean"][..., None]) * d["rstd"][..., None]
        dy = d["dy"].view(N, P, G, D).permute(0, 2, 1, 3).reshape(N, G, n)
        dh = dy * _gate64(xh * wb[0] + wb[1], c["act"])[1]
        g = dh * wb[0]
        dx = (n * g - g.sum(2, keepdim=True) - xh * (g * xh).sum(2, keepdim=True)) * (d["rstd"][..., None] / n)
        sums = [v.view(N, G, P, D).sum((0, 2)).reshape(-1) for v in (dh * xh, dh)]
        return back(dx), sums[0], sums[1]
    if op == "f8_fwd":
        h = torch.mm(_value64(s["wq"], s["we"], c["I"]), _held64(d["x"], "e4m3").t()).t()
        if c["bias"]:
            h = h + d["b"]
        y = _gate64(h, c["act"])[0]
        if c["res"]:
            y = y + d["res"]
        return (y, h) if c["save"] else y
    if op == "f8_bwd_input":
        dx = torch.mm(_value64(s["wq"], s["we"], c["O"]), _held64(d["dy"], c["fmt"]).t()).t()
        return dx if s["pre"] is None else dx * _gate64(d["pre"], c["act"])[1]
    dw = torch.mm(_value64(s["xq"], s["xe"], c["M"]), _held64(d["dy"].t().contiguous(), c["fmt"]).t()).t()
    return dw, torch.ones(c["M"], device="cuda").double() @ d["dy"]
