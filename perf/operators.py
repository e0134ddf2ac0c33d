"""The operators of a training step around the sparse gradient exchange, as measured cases.

A worker's step is: linear layers forward (product, bias, activation, residual in one call), the softmax cross-entropy with
the gradient of its logits, the layers backward (input, weight and bias gradients, the latter in fp32 where the compression
takes them), and - on the server, once the pushes are summed - one AdamW step over all tensors of a shard, its moments kept
in 32 or in 8 bits.  Each case is one such call; `run` computes it with elementary torch operations in 32 bits, or, where
`own` is set, through this repository's library.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_ITEM = {"bf16": 2, "fp16": 2, "fp32": 4}
_BLOCK = 128                       # consecutive elements that share a window of exponents in the 8-bit moments
_IGNORE = -100

# the six and the twelve tensors of the two models whose gradients the benchmark compresses, in elements
_MNIST = "3211264,4096,16777216,4096,40960,10"
_NMT = "42500000,42500000,42500000,85000" + ",1500000,1000000" * 4


# ------------------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # one input through a 4096 x 4096 layer: the call of a server that answers one request at a time
        {"name": "forward one row", "op": "forward", "m": 1, "n": 4096, "k": 4096, "dtype": "bf16", "out": "bf16", "act": "relu",
         "layout": "in_out", "bias": True, "residual": False, "pre": False},
        # the first layer of the MNIST-shaped model on a batch of 80, pre-activation kept for the backward pass
        {"name": "forward batch of 80", "op": "forward", "m": 80, "n": 4096, "k": 784, "dtype": "bf16", "out": "bf16", "act": "relu",
         "layout": "in_out", "bias": True, "residual": False, "pre": True},
        # the output projection of the translation model: 80 sentences of 50 tokens onto 85000 words; rows of 1000 bytes
        {"name": "forward vocabulary", "op": "forward", "m": 4000, "n": 85000, "k": 500, "dtype": "bf16", "out": "bf16", "act": "none",
         "layout": "in_out", "bias": True, "residual": False, "pre": False},
        # a large batch through a square layer with a skip connection
        {"name": "forward large", "op": "forward", "m": 16384, "n": 4096, "k": 4096, "dtype": "bf16", "out": "bf16", "act": "gelu",
         "layout": "out_in", "bias": True, "residual": True, "pre": True},
        # the last layer of the MNIST-shaped model backward: ten classes
        {"name": "backward ten classes", "op": "backward", "m": 80, "n": 10, "k": 4096, "dtype": "bf16", "grads": "fp32", "act": "none",
         "layout": "in_out"},
        # a recurrent block's input matrix backward over 80 sentences of 50 tokens, half precision throughout
        {"name": "backward recurrent block", "op": "backward", "m": 4000, "n": 1000, "k": 1500, "dtype": "fp16", "grads": "fp16", "act": "silu",
         "layout": "in_out"},
        # a large batch through a square layer backward, the weight gradient in fp32 as the compression takes it
        {"name": "backward large", "op": "backward", "m": 8192, "n": 4096, "k": 4096, "dtype": "bf16", "grads": "fp32", "act": "relu",
         "layout": "in_out"},
        # the loss of a batch of 80 over ten classes
        {"name": "loss ten classes", "op": "loss", "rows": 80, "classes": 10, "dtype": "fp32", "ignored": 0.0},
        # the loss over the vocabulary, with padding positions that carry no target
        {"name": "loss vocabulary", "op": "loss", "rows": 4000, "classes": 85000, "dtype": "bf16", "ignored": 0.1},
        # the optimiser step of the MNIST-shaped model: six tensors, moments in 8 bits, 16-bit copy of the weights written too
        {"name": "adamw 8 bits small model", "op": "adamw", "sizes": _MNIST, "bits": 8, "param": "fp32", "grad": "fp32", "copy": True},
        # the translation model's twelve tensors, moments in 32 bits and in 8
        {"name": "adamw 32 bits", "op": "adamw", "sizes": _NMT, "bits": 32, "param": "fp32", "grad": "fp32", "copy": False},
        {"name": "adamw 8 bits", "op": "adamw", "sizes": _NMT, "bits": 8, "param": "fp32", "grad": "bf16", "copy": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "loss", "adamw"])
    if op in ("forward", "backward"):
        while True:
            m, n, k = _log(rng, 1, 16384), _log(rng, 10, 85000), _log(rng, 16, 4096)
            # most widths in use are multiples of eight; the others have rows that start at any even address
            n, k = (v if rng.random() < 0.4 else max(8, v // 8 * 8) for v in (n, k))
            cost = m * n * k * (1 if op == "forward" else 2)
            if cost <= (1 << 38) and m * n <= 340_000_000 // (1 if op == "forward" else 4) and n * k <= 1 << 26:
                break
        act = rng.choice(["none", "relu", "gelu", "silu"])
        case = {"op": op, "m": m, "n": n, "k": k, "dtype": rng.choice(["bf16", "fp16"]), "act": act, "layout": rng.choice(["in_out", "out_in"])}
        if op == "forward":
            case.update(out=rng.choice([case["dtype"], case["dtype"], "fp32"]), bias=rng.random() < 0.7, residual=rng.random() < 0.4, pre=rng.random() < 0.5)
        else:
            # where the activation's derivative is not 0 or 1 the two products take it rounded to 16 bits, and so is what they give
            case["grads"] = rng.choice([case["dtype"], "fp32"]) if act in ("none", "relu") else case["dtype"]
        return case
    if op == "loss":
        while True:
            rows, classes = _log(rng, 1, 60000), _log(rng, 2, 200000)
            if rows * classes <= 340_000_000 // 2:
                break
        return {"op": op, "rows": rows, "classes": classes, "dtype": rng.choice(["bf16", "fp16", "fp32"]), "ignored": rng.choice([0.0, 0.05, 0.3])}
    count, total = _log(rng, 1, 400), _log(rng, 2000, 130_000_000)
    cuts = sorted(rng.random() for _ in range(count - 1))
    sizes = [max(1, int((b - a) * total)) for a, b in zip([0.0] + cuts, cuts + [1.0])]
    return {"op": op, "sizes": ",".join(map(str, sizes)), "bits": rng.choice([8, 32]), "param": rng.choice(["fp32", "fp32", "bf16"]),
            "grad": rng.choice(["fp32", "bf16"]), "copy": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------------------- the inputs

def _randn(gen, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device=gen.device) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"forward": _prepare_forward, "backward": _prepare_backward, "loss": _prepare_loss, "adamw": _prepare_adamw}[case["op"]](case, gen)


def _linear_inputs(case, gen):
    m, n, k, dt = case["m"], case["n"], case["k"], _DT[case["dtype"]]
    s = {"case": case, "x": _randn(gen, m, k, dtype=dt), "w": _randn(gen, *((k, n) if case["layout"] == "in_out" else (n, k)), scale=k ** -0.5, dtype=dt)}
    if own:
        from paper_1704_05021_b200 import training
        s["session"] = training.LinearSession(k, n, m, dtype=dt, activation=case["act"], w_layout=case["layout"], device="cuda")
    return s


def _prepare_forward(case, gen):
    m, n, dt = case["m"], case["n"], _DT[case["dtype"]]
    s = _linear_inputs(case, gen)
    s["bias"] = _randn(gen, n, scale=0.1) if case["bias"] else None
    s["residual"] = _randn(gen, m, n, dtype=dt) if case["residual"] else None
    s["y"] = torch.empty(m, n, dtype=_DT[case["out"]], device="cuda")
    s["pre"] = torch.empty(m, n, dtype=dt, device="cuda") if case["pre"] else None
    return s


def _prepare_backward(case, gen):
    m, n, k, dt = case["m"], case["n"], case["k"], _DT[case["dtype"]]
    s = _linear_inputs(case, gen)
    s["dy"] = _randn(gen, m, n, scale=1e-2, dtype=dt)
    s["pre"] = _randn(gen, m, n, dtype=dt) if case["act"] != "none" else None
    s["dx"] = torch.empty(m, k, dtype=dt, device="cuda")
    s["dw"] = torch.empty_like(s["w"], dtype=_DT[case["grads"]])
    s["db"] = torch.empty(n, dtype=torch.float32, device="cuda")
    return s


def _prepare_loss(case, gen):
    rows, classes, dt = case["rows"], case["classes"], _DT[case["dtype"]]
    logits = _randn(gen, rows, classes, scale=2.0, dtype=dt)
    targets = torch.randint(classes, (rows,), generator=gen, device="cuda")
    targets[torch.rand(rows, generator=gen, device="cuda") < case["ignored"]] = _IGNORE
    s = {"case": case, "logits": logits, "targets": targets, "scale": (1024.0 if case["dtype"] == "fp16" else 1.0) / rows}   # (half precision: the usual loss scale)
    s["loss"], s["lse"] = (torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(2))
    s["grad"] = torch.empty_like(logits)
    if own:
        from paper_1704_05021_b200 import training
        s["loss_of"] = training.cross_entropy
    return s


def _cut(flat, sizes):
    return list(torch.split(flat, sizes))


def _prepare_adamw(case, gen):
    sizes = [int(t) for t in case["sizes"].split(",")]
    blocks = [-(-n // _BLOCK) for n in sizes]
    total, eight = sum(sizes), case["bits"] == 8
    s = {"case": case, "lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "step": 1000, "seed": 12345}
    s["decay"] = [0.01 if n > 5000 else 0.0 for n in sizes]              # matrices decay, biases do not
    # one flat vector each, as the gradient exchange has them; the tensors are pieces of it, at whatever offsets they get
    flat = {"params": _randn(gen, total, scale=0.02, dtype=_DT[case["param"]]), "grads": _randn(gen, total, scale=1e-3, dtype=_DT[case["grad"]])}
    if case["copy"]:
        flat["copies"] = torch.empty(total, dtype=torch.bfloat16, device="cuda")
    m = _randn(gen, total, scale=3e-4)
    v = torch.rand(total, generator=gen, device="cuda") * 2e-6 + 1e-8
    if eight:
        for name, x in (("m", m), ("v", torch.sqrt(v))):
            half = torch.full((max(sizes),), 1 << 15, dtype=torch.int32, device="cuda")
            pairs = [_encode(t, half[:t.numel()], name == "v") for t in torch.split(x, sizes)]
            flat[name] = torch.cat([t[0][:n].view(torch.uint8) for t, n in zip(pairs, sizes)]).view(torch.float8_e4m3fn)
            flat[name + "_scale"] = torch.cat([t[1] for t in pairs])
    else:
        flat["m"], flat["v"] = m, v
    s["flat"] = flat
    s.update({name: _cut(t, blocks if name.endswith("_scale") else sizes) for name, t in flat.items()})
    if own:
        from paper_1704_05021_b200 import training
        s["session"] = training.AdamWSession(s["params"], s["grads"], s["m"], s["v"], s.get("m_scale"), s.get("v_scale"),
                                             copies=s.get("copies"), weight_decay=s["decay"])
    return s


# ------------------------------------------------------------------------------------------------------------- the calls

def run(s):
    return {"forward": _forward, "backward": _backward, "loss": _loss, "adamw": _adamw}[s["case"]["op"]](s)


def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    g = 1.0 / (1.0 + torch.exp(-z))
    return g * (1.0 + z * (1.0 - g))


def _forward(s):
    case = s["case"]
    if own:
        s["session"].forward(s["x"], s["w"], s["bias"], s["residual"], out=s["y"], pre=s["pre"])
        return {"y": s["y"], "pre": s["pre"]}
    w = s["w"].float()
    z = s["x"].float() @ (w if case["layout"] == "in_out" else w.t())
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(_DT[case["out"]]), "pre": z.to(_DT[case["dtype"]]) if case["pre"] else None}


def _backward(s):
    case = s["case"]
    if own:
        s["session"].backward(s["dy"], s["x"], s["w"], s["pre"], dx=s["dx"], dw=s["dw"], db=s["db"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    dz, x, w = s["dy"].float(), s["x"].float(), s["w"].float()
    if s["pre"] is not None:
        dz = dz * _act_slope(s["pre"].float(), case["act"])
    dx = dz @ (w.t() if case["layout"] == "in_out" else w)
    dw = x.t() @ dz if case["layout"] == "in_out" else dz.t() @ x
    return {"dx": dx.to(_DT[case["dtype"]]), "dw": dw.to(_DT[case["grads"]]), "db": dz.sum(0)}


def _loss(s):
    if own:
        s["loss_of"](s["logits"], s["targets"], loss=s["loss"], lse=s["lse"], grad=s["grad"], grad_scale=s["scale"], ignore_index=_IGNORE)
        return {"loss": s["loss"], "lse": s["lse"], "grad": s["grad"]}
    x, t = s["logits"].float(), s["targets"]
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    live = t != _IGNORE
    at = torch.where(live, t, torch.zeros_like(t)).unsqueeze(1)
    loss = torch.where(live, lse - x.gather(1, at).squeeze(1), torch.zeros_like(lse))
    g = e / total
    g.scatter_add_(1, at, torch.full_like(total, -1.0))
    g = g * (live.float() * s["scale"]).unsqueeze(1)
    return {"loss": loss, "lse": lse, "grad": g.to(s["logits"].dtype)}


# The 8-bit moments.  The first moment and the square root of the second are held in fp8 (1 sign, 4 exponent, 3 mantissa bits),
# in units of a power of two that a block of 128 consecutive elements shares and that puts the block's largest magnitude into
# [128, 256).  A magnitude is rounded up or down to one of its neighbours by a 16-bit random number, so that what is held is
# right on average; a positive root is never rounded to zero, and what is not finite is held as NaN.

def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % _BLOCK)).view(-1, _BLOCK)


def _encode(x, random16, positive):
    x = _blocks(x)
    size = x.abs()
    exponent = ((size.view(torch.int32).amax(1, keepdim=True) >> 23) - 7).clamp(min=1)
    scale, inverse = (exponent << 23).view(torch.float32), ((254 - exponent) << 23).view(torch.float32)
    y = size * inverse
    # in units of the last bit kept, times 2^20: normal numbers by their bits, those below 2^-6 by the fixed step there
    units = torch.where(y >= 2.0 ** -6, y.view(torch.int32) - (120 << 23), (y + 2.0 ** -6).view(torch.int32) - (121 << 23))
    code = ((units + (_blocks(random16) << 4)) >> 20).clamp(max=127)
    code = torch.where(y.isfinite(), code, torch.full_like(code, 127))
    if positive:
        code = torch.where(size > 0, code.clamp(min=1), code)
    code = code | ((x.view(torch.int32) < 0).to(torch.int32) << 7)
    return code.reshape(-1).to(torch.uint8).view(torch.float8_e4m3fn), scale.reshape(-1)


def _decode(held, scale):
    return (_blocks(held.float()) * scale.unsqueeze(1)).reshape(-1)[:held.numel()]


def _i32(x):
    x &= 0xFFFFFFFF
    return x - (1 << 32) if x >> 31 else x


def _random(n, seed, tensor):
    """Two 16-bit random numbers for each element of a tensor: the halves of a 32-bit mix of its index and the seed."""
    x = torch.arange(n, dtype=torch.int32, device="cuda") * _i32(0x9E3779B9) + _i32(seed + tensor * 0x85EBCA77)
    x = (x ^ ((x >> 16) & 0xFFFF)) * _i32(0x7FEB352D)
    x = (x ^ ((x >> 15) & 0x1FFFF)) * _i32(0x846CA68B)
    x = x ^ ((x >> 16) & 0xFFFF)
    return (x >> 16) & 0xFFFF, x & 0xFFFF


def _adamw_one(s, t):
    """One tensor's step, every operation rounded to fp32 in this order; parameters and moments are updated in place."""
    p, eight = s["params"][t], s["case"]["bits"] == 8
    m = _decode(s["m"][t], s["m_scale"][t]) if eight else s["m"][t]
    v = _decode(s["v"][t], s["v_scale"][t]).square() if eight else s["v"][t]
    g = s["grads"][t].float()
    m = m * s["beta1"] + g * (1.0 - s["beta1"])
    v = v * s["beta2"] + (g * (1.0 - s["beta2"])) * g
    root = torch.sqrt(v)
    below = root * (1.0 / math.sqrt(1.0 - s["beta2"] ** s["step"])) + s["eps"]
    q = p.float() * (1.0 - s["lr"] * s["decay"][t]) - (m / below) * (s["lr"] / (1.0 - s["beta1"] ** s["step"]))
    p.copy_(q)
    if "copies" in s:
        s["copies"][t].copy_(q)
    if eight:
        high, low = _random(m.numel(), s["seed"], t)
        (held_m, scale_m), (held_v, scale_v) = _encode(m, high, False), _encode(root, low, True)
        s["m"][t].copy_(held_m[:m.numel()]), s["m_scale"][t].copy_(scale_m)
        s["v"][t].copy_(held_v[:m.numel()]), s["v_scale"][t].copy_(scale_v)
    else:
        s["m"][t].copy_(m), s["v"][t].copy_(v)


def _adamw(s):
    if own:
        s["session"].step(step=s["step"], lr=s["lr"], beta1=s["beta1"], beta2=s["beta2"], eps=s["eps"], seed=s["seed"])
    else:
        list(map(lambda t: _adamw_one(s, t), range(len(s["params"]))))
    return {name: s["flat"][name] for name in ("params", "copies", "m", "v", "m_scale", "v_scale") if name in s["flat"]}


def work(case):
    op = case["op"]
    if op in ("forward", "backward"):
        m, n, k, e = case["m"], case["n"], case["k"], _ITEM[case["dtype"]]
        if op == "forward":
            b = e * (m * k + k * n) + _ITEM[case["out"]] * m * n + (4 * n if case["bias"] else 0) + e * m * n * (int(case["residual"]) + int(case["pre"]))
            return {"bytes": b, "flops": 2 * m * n * k}
        b = e * (m * n * (2 if case["act"] != "none" else 1) + 2 * m * k + k * n) + _ITEM[case["grads"]] * k * n + 4 * n
        return {"bytes": b, "flops": 4 * m * n * k}
    if op == "loss":
        cells = case["rows"] * case["classes"]
        return {"bytes": 2 * _ITEM[case["dtype"]] * cells + 16 * case["rows"], "flops": 6 * cells}
    n = sum(int(t) for t in case["sizes"].split(","))
    state = 16 if case["bits"] == 32 else 4 + 16 / _BLOCK
    return {"bytes": n * (2 * _ITEM[case["param"]] + _ITEM[case["grad"]] + state + (2 if case["copy"] else 0)), "flops": 16 * n}


# ------------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"forward": _exact_forward, "backward": _exact_backward, "loss": _exact_loss, "adamw": _exact_adamw}[case["op"]](s)


def _exact_forward(s):
    case = s["case"]
    weight = s["w"].double() if case["layout"] == "out_in" else s["w"].double().T
    z = torch.nn.functional.linear(s["x"].double(), weight, None if s["bias"] is None else s["bias"].double())
    y = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]](z)
    if s["residual"] is not None:
        y = y + s["residual"]
    return {"y": y, "pre": z if case["pre"] else None}


def _exact_backward(s):
    case = s["case"]
    x, w = (s[name].double().requires_grad_() for name in ("x", "w"))
    dz = s["dy"].double()
    if s["pre"] is not None:
        z = s["pre"].double().requires_grad_()
        with torch.enable_grad():
            y = {"relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]](z)
        dz, = torch.autograd.grad(y, z, dz)
    with torch.enable_grad():
        z = torch.nn.functional.linear(x, w if case["layout"] == "out_in" else w.T)
    dx, dw = torch.autograd.grad(z, (x, w), dz)
    return {"dx": dx, "dw": dw, "db": dz.sum(0)}


def _exact_loss(s):
    z = s["logits"].double()
    lse = torch.logsumexp(z, 1)
    live = s["targets"] != _IGNORE
    loss = torch.nn.functional.nll_loss(z - lse[:, None], s["targets"], ignore_index=_IGNORE, reduction="none")
    grad = torch.softmax(z, 1)
    rows = torch.arange(len(z), device=z.device)[live]
    grad[rows, s["targets"][live]] -= 1.0
    return {"loss": loss, "lse": lse, "grad": grad * (live.double() * s["scale"])[:, None]}


def _exact_adamw(s):
    eight, step = s["case"]["bits"] == 8, s["step"]
    out = {name: [] for name in ("params", "m", "v") + (("copies",) if "copies" in s else ()) + (("m_scale", "v_scale") if eight else ())}

    def held(x):
        top = torch.nn.functional.pad(x.abs(), (0, -len(x) % _BLOCK)).view(-1, _BLOCK).amax(1)
        unit = torch.exp2(torch.floor(torch.log2(top)) - 7.0)
        return x / unit.repeat_interleave(_BLOCK)[:len(x)], unit

    for t, p in enumerate(s["params"]):
        g, m, v = s["grads"][t].double(), s["m"][t].double(), s["v"][t].double()
        if eight:
            wide = [s[name][t].double().repeat_interleave(_BLOCK)[:len(m)] for name in ("m_scale", "v_scale")]
            m, v = m * wide[0], (v * wide[1]) ** 2
        m = torch.lerp(g, m, s["beta1"])
        v = torch.lerp(g * g, v, s["beta2"])
        hat_m, hat_v = m / (1.0 - s["beta1"] ** step), v / (1.0 - s["beta2"] ** step)
        q = p.double() - s["lr"] * (hat_m / (hat_v.sqrt() + s["eps"]) + s["decay"][t] * p.double())
        out["params"].append(q)
        if "copies" in out:
            out["copies"].append(q)
        if eight:
            (m, unit_m), (v, unit_v) = held(m), held(v.sqrt())
            out["m_scale"].append(unit_m)
            out["v_scale"].append(unit_v)
        out["m"].append(m)
        out["v"].append(v)
    return {name: torch.cat(parts) for name, parts in out.items()}
