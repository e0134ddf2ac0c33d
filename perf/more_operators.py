"""The layers of a language model around its linear layers, as measured cases.

What stands between the tokens and the loss beside plain linear layers: the embedding lookup with its gradient by sorted tokens (the
largest tensors of the translation model whose gradients the benchmark compresses are embeddings), layer norm forward and backward, a
gated linear recurrence over packed sequences forward (down to single tokens) and backward, and the gated feed-forward block, both
projections, activation and product in one call, forward and backward.  Each case is one such call; `run` computes it with elementary torch
operations in 32 bits, or, where `own` is set, through this repository's library.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_ITEM = {"bf16": 2, "fp16": 2, "fp32": 4}
_IGNORE = -100
_EPS = 1e-5
_MARK = 64                         # steps between the states that the recurrence keeps for its backward pass


# ------------------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # the encoder's input: 80 sentences of 50 tokens out of 85000 words, rows of 1000 bytes, a tenth of the positions padding
        {"name": "embedding forward batch", "op": "embed", "tokens": 4000, "vocab": 85000, "width": 500, "table": "bf16", "out": "bf16", "ignored": 0.1},
        # its gradient, in fp32 as the compression takes it: nearly all of it is the zeros of words that do not occur
        {"name": "embedding backward batch", "op": "embed_back", "tokens": 4000, "vocab": 85000, "width": 500, "dtype": "bf16", "grads": "fp32",
         "ignored": 0.1},
        # a large batch over a smaller vocabulary: every frequent word occurs thousands of times
        {"name": "embedding backward large", "op": "embed_back", "tokens": 131072, "vocab": 32000, "width": 1024, "dtype": "bf16", "grads": "fp32",
         "ignored": 0.0},
        # one row: the call of a server that answers one request at a time
        {"name": "norm forward one row", "op": "norm", "rows": 1, "width": 4096, "dtype": "bf16"},
        # a large batch
        {"name": "norm forward large", "op": "norm", "rows": 32768, "width": 4096, "dtype": "bf16"},
        # a recurrent block's norm backward over 80 sentences of 50 tokens, with the gradient that comes past the norm
        {"name": "norm backward batch", "op": "norm_back", "rows": 4000, "width": 1000, "dtype": "fp16", "add": True},
        # one token for each of 64 sequences
        {"name": "recurrence one step", "op": "scan", "rows": 64, "sequences": 64, "width": 1024, "dtype": "bf16", "ragged": False, "keep": False},
        # one long document
        {"name": "recurrence forward long", "op": "scan", "rows": 65536, "sequences": 1, "width": 1024, "dtype": "bf16", "ragged": False, "keep": True},
        # a packed batch of sentences of many lengths, backward
        {"name": "recurrence backward ragged", "op": "scan_back", "rows": 16000, "sequences": 80, "width": 1000, "dtype": "bf16", "ragged": True},
        # one row through both projections
        {"name": "gated forward one row", "op": "gated", "m": 1, "n": 4096, "k": 2048, "dtype": "bf16", "act": "silu", "layout": "in_out", "bias": False,
         "pre": False},
        # a large batch, pre-activations kept for the backward pass
        {"name": "gated forward large", "op": "gated", "m": 8192, "n": 5632, "k": 2048, "dtype": "bf16", "act": "silu", "layout": "out_in", "bias": True,
         "pre": True},
        # a batch backward
        {"name": "gated backward", "op": "gated_back", "m": 4000, "n": 2048, "k": 1000, "dtype": "bf16", "act": "gelu", "layout": "in_out"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Most widths in use are multiples of eight; the others have rows that start at any multiple of the element's size."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.35 else max(8, n // 8 * 8)


def draw(rng):
    op = rng.choice(["embed", "embed_back", "norm", "norm_back", "scan", "scan_back", "gated", "gated_back"])
    if op in ("embed", "embed_back"):
        while True:
            tokens, vocab, width = _log(rng, 1, 131072), _log(rng, 64, 200000), _width(rng, 8, 4096)
            if tokens * width <= 131072 * 1024 // 2 and vocab * width <= 85000 * 500:
                break
        ignored = rng.choice([0.0, 0.1, 0.5])
        if op == "embed":
            table = rng.choice(["bf16", "fp16", "fp32"])
            return {"op": op, "tokens": tokens, "vocab": vocab, "width": width, "table": table, "ignored": ignored,
                    "out": rng.choice([table, table, "fp32"]) if table != "fp32" else rng.choice(["bf16", "fp16", "fp32"])}
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        return {"op": op, "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "grads": rng.choice(["fp32", "fp32", dtype]), "ignored": ignored}
    if op in ("norm", "norm_back"):
        while True:
            rows, width = _log(rng, 1, 65536), _width(rng, 16, 16384)
            if rows * width <= 32768 * 4096 // 2:
                break
        case = {"op": op, "rows": rows, "width": width, "dtype": rng.choice(["bf16", "fp16", "fp32"])}
        if op == "norm_back":
            case["add"] = rng.random() < 0.5
        return case
    if op in ("scan", "scan_back"):
        while True:
            rows, sequences, width = _log(rng, 1, 65536), _log(rng, 1, 512), _width(rng, 8, 4096)
            if rows * width <= 65536 * 1024 // 2 and sequences <= rows:
                break
        ragged = rng.random() < 0.6
        if not ragged:
            rows -= rows % sequences
        case = {"op": op, "rows": rows, "sequences": sequences, "width": width, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "ragged": ragged}
        if op == "scan":
            case["keep"] = rng.random() < 0.5
        return case
    while True:
        m, n, k = _log(rng, 1, 8192), _width(rng, 16, 8192), _width(rng, 16, 4096)
        if 2 * m * n * k * (1 if op == "gated" else 2) <= 1 << 36 and n * k <= 1 << 24:
            break
    case = {"op": op, "m": m, "n": n, "k": k, "dtype": rng.choice(["bf16", "fp16"]), "act": rng.choice(["none", "relu", "gelu", "silu"]),
            "layout": rng.choice(["in_out", "out_in"])}
    if op == "gated":
        case.update(bias=rng.random() < 0.5, pre=rng.random() < 0.5)
    return case


# ------------------------------------------------------------------------------------------------------------- the inputs

def _randn(gen, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device=gen.device) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"embed": _prepare_embed, "embed_back": _prepare_embed_back, "norm": _prepare_norm, "norm_back": _prepare_norm_back, "scan": _prepare_scan,
            "scan_back": _prepare_scan_back, "gated": _prepare_gated, "gated_back": _prepare_gated_back}[case["op"]](case, gen)


def _tokens(case, gen):
    """Words of a vocabulary sorted by frequency: the chance of word i falls like 1 / i.  Padding positions carry no word."""
    u = torch.rand(case["tokens"], generator=gen, device="cuda", dtype=torch.float64)
    t = (torch.exp(u * math.log(case["vocab"] + 1.0)) - 1.0).long().clamp(max=case["vocab"] - 1)
    return torch.where(torch.rand(case["tokens"], generator=gen, device="cuda") < case["ignored"], torch.full_like(t, _IGNORE), t)


def _embed_state(case, gen):
    s = {"case": case, "tokens": _tokens(case, gen), "scale": math.sqrt(case["width"])}
    if own:
        from paper_1704_05021_b200 import layers
        s["session"] = layers.EmbeddingSession(case["vocab"], case["width"], case["tokens"], device="cuda")
    return s


def _prepare_embed(case, gen):
    s = _embed_state(case, gen)
    s["table"] = _randn(gen, case["vocab"], case["width"], scale=0.02, dtype=_DT[case["table"]])
    s["y"] = torch.empty(case["tokens"], case["width"], dtype=_DT[case["out"]], device="cuda")
    return s


def _prepare_embed_back(case, gen):
    s = _embed_state(case, gen)
    s["dy"] = _randn(gen, case["tokens"], case["width"], scale=1e-2, dtype=_DT[case["dtype"]])
    s["dtable"] = torch.empty(case["vocab"], case["width"], dtype=_DT[case["grads"]], device="cuda")
    return s


def _norm_state(case, gen):
    rows, width, dt = case["rows"], case["width"], _DT[case["dtype"]]
    # rows of different sizes around means that are not zero
    level = _randn(gen, rows, 1)
    s = {"case": case, "x": (level + _randn(gen, rows, width) * (0.5 + level.abs())).to(dt), "weight": 1.0 + _randn(gen, width, scale=0.1)}
    if own:
        from paper_1704_05021_b200 import layers
        s["session"] = layers.LayerNormSession(width, rows, dtype=dt, eps=_EPS, device="cuda")
    return s


def _prepare_norm(case, gen):
    s = _norm_state(case, gen)
    s["bias"] = _randn(gen, case["width"], scale=0.1)
    s["y"] = torch.empty_like(s["x"])
    s["mean"], s["rstd"] = (torch.empty(case["rows"], dtype=torch.float32, device="cuda") for _ in range(2))
    return s


def _prepare_norm_back(case, gen):
    s = _norm_state(case, gen)
    x = s["x"].double()
    mean = x.mean(1)
    s["mean"], s["rstd"] = mean.float(), ((x - mean[:, None]).square().mean(1) + _EPS).rsqrt().float()
    s["dy"] = _randn(gen, *s["x"].shape, scale=1e-2, dtype=s["x"].dtype)
    s["add"] = _randn(gen, *s["x"].shape, scale=1e-2, dtype=s["x"].dtype) if case["add"] else None
    s["dx"] = torch.empty_like(s["x"])
    s["dweight"], s["dbias"] = (torch.empty(case["width"], dtype=torch.float32, device="cuda") for _ in range(2))
    return s


def _scan_state(case, gen):
    rows, count, width, dt = case["rows"], case["sequences"], case["width"], _DT[case["dtype"]]
    # gates that remember for a few to some hundred steps
    s = {"case": case, "gate": (2.0 + _randn(gen, rows, width, scale=1.5)).to(dt), "value": _randn(gen, rows, width, dtype=dt), "offsets": None}
    if case["ragged"]:
        # lengths from none to a few times the mean; some rows behind the last sequence belong to nobody
        cuts = torch.rand(count, generator=gen, device="cuda", dtype=torch.float64).sort().values
        ends = (cuts * (rows + 1)).long().clamp(max=rows - rows // 50)
        ends[-1] = rows - rows // 50
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), ends])
    s["h0"] = _randn(gen, count, width, scale=0.3)
    return s


def _prepare_scan(case, gen):
    s = _scan_state(case, gen)
    rows, count, width = case["rows"], case["sequences"], case["width"]
    s["y"], s["h_last"] = torch.zeros_like(s["value"]), torch.empty(count, width, dtype=torch.float32, device="cuda")
    if own:
        from paper_1704_05021_b200 import layers
        s["call"] = layers.recurrence_forward
        s["marks"] = layers.recurrence_marks(rows, count, width, device="cuda") if case["keep"] else None
    return s


def _prepare_scan_back(case, gen):
    s = _scan_state(case, gen)
    rows, count, width = case["rows"], case["sequences"], case["width"]
    s["dy"], s["dh_last"] = _randn(gen, rows, width, scale=1e-2, dtype=s["value"].dtype), _randn(gen, count, width, scale=1e-2)
    s["dgate"], s["dvalue"] = torch.zeros_like(s["gate"]), torch.zeros_like(s["value"])
    s["dh0"] = torch.empty(count, width, dtype=torch.float32, device="cuda")
    if own:
        from paper_1704_05021_b200 import layers
        s["call"] = layers.recurrence_backward
        s["marks"] = layers.recurrence_marks(rows, count, width, device="cuda")
        layers.recurrence_forward(s["gate"], s["value"], out=torch.empty_like(s["value"]), offsets=s["offsets"], sequences=count, h0=s["h0"],
                                  marks=s["marks"])
    return s


def _gated_state(case, gen):
    m, n, k, dt = case["m"], case["n"], case["k"], _DT[case["dtype"]]
    s = {"case": case, "x": _randn(gen, m, k, dtype=dt),
         "w": _randn(gen, *((k, 2 * n) if case["layout"] == "in_out" else (2 * n, k)), scale=k ** -0.5, dtype=dt)}
    if own:
        from paper_1704_05021_b200 import layers
        s["session"] = layers.GatedLinearSession(k, n, m, dtype=dt, activation=case["act"], w_layout=case["layout"], device="cuda")
    return s


def _prepare_gated(case, gen):
    s = _gated_state(case, gen)
    m, n, dt = case["m"], case["n"], _DT[case["dtype"]]
    s["bias"] = _randn(gen, 2 * n, scale=0.1) if case["bias"] else None
    s["y"] = torch.empty(m, n, dtype=dt, device="cuda")
    s["pre"] = torch.empty(m, 2 * n, dtype=dt, device="cuda") if case["pre"] else None
    return s


def _prepare_gated_back(case, gen):
    s = _gated_state(case, gen)
    m, n, k, dt = case["m"], case["n"], case["k"], _DT[case["dtype"]]
    s["dy"] = _randn(gen, m, n, scale=1e-2, dtype=dt)
    s["pre"] = _randn(gen, m, 2 * n, dtype=dt)
    s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    s["db"] = torch.empty(2 * n, dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------------- the calls

def run(s):
    return {"embed": _embed, "embed_back": _embed_back, "norm": _norm, "norm_back": _norm_back, "scan": _scan, "scan_back": _scan_back, "gated": _gated,
            "gated_back": _gated_back}[s["case"]["op"]](s)


def _embed(s):
    if own:
        s["session"].forward(s["table"], s["tokens"], out=s["y"], scale=s["scale"], ignore_index=_IGNORE)
        return {"y": s["y"]}
    live = s["tokens"] != _IGNORE
    rows = s["table"][torch.where(live, s["tokens"], torch.zeros_like(s["tokens"]))].float() * s["scale"]
    return {"y": torch.where(live[:, None], rows, torch.zeros_like(rows)).to(_DT[s["case"]["out"]])}


def _embed_back(s):
    case = s["case"]
    if own:
        s["session"].backward(s["dy"], s["tokens"], s["dtable"], scale=s["scale"], ignore_index=_IGNORE)
        return {"dtable": s["dtable"]}
    live = s["tokens"] != _IGNORE
    rows = torch.where(live[:, None], s["dy"].float() * s["scale"], torch.zeros((), device="cuda"))
    total = torch.zeros(case["vocab"], case["width"], device="cuda")
    total.index_add_(0, torch.where(live, s["tokens"], torch.zeros_like(s["tokens"])), rows)
    return {"dtable": total.to(_DT[case["grads"]])}


def _norm(s):
    if own:
        s["session"].forward(s["x"], s["weight"], s["bias"], out=s["y"], mean=s["mean"], rstd=s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    x = s["x"].float()
    mean = x.sum(1, keepdim=True) * (1.0 / x.shape[1])
    x = x - mean
    rstd = 1.0 / torch.sqrt((x * x).sum(1, keepdim=True) * (1.0 / x.shape[1]) + _EPS)
    return {"y": (x * rstd * s["weight"] + s["bias"]).to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _norm_back(s):
    if own:
        s["session"].backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], dx=s["dx"], add=s["add"], dweight=s["dweight"], dbias=s["dbias"])
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    dy, share = s["dy"].float(), 1.0 / s["x"].shape[1]
    hat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"]
    dx = (g - g.sum(1, keepdim=True) * share - hat * ((g * hat).sum(1, keepdim=True) * share)) * s["rstd"][:, None]
    if s["add"] is not None:
        dx = dx + s["add"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * hat).sum(0), "dbias": dy.sum(0)}


def _spans(s):
    """First and last row of every sequence, and which sequence each row belongs to (the number of sequences where none)."""
    rows, count = s["case"]["rows"], s["case"]["sequences"]
    offsets = s["offsets"] if s["offsets"] is not None else torch.arange(count + 1, device="cuda") * (rows // count)
    row = torch.arange(rows, device="cuda")
    return offsets, torch.searchsorted(offsets[1:].contiguous(), row, right=True), row


def _scan_rows(keep, add):
    """h[t] = keep[t] h[t-1] + add[t] from h = 0 over all rows, by doubling: keep is 0 where a sequence begins."""
    step = 1
    while step < len(add):
        add = torch.cat([add[:step], torch.addcmul(add[step:], keep[step:], add[:-step])])
        keep = torch.cat([keep[:step], keep[step:] * keep[:-step]])
        step *= 2
    return add


def _states(s):
    """Every row's state, the state before it, and the gate's two weights."""
    offsets, owner, row = _spans(s)
    count = s["case"]["sequences"]
    gate, value = s["gate"].float(), s["value"].float()
    keep, take = 1.0 / (1.0 + torch.exp(-gate)), 1.0 / (1.0 + torch.exp(gate))
    inside = (owner < count)[:, None]
    whose = owner.clamp(max=count - 1)
    first = (row == offsets[whose])[:, None]
    begin = s["h0"][whose]
    h = _scan_rows(torch.where(first | ~inside, torch.zeros_like(keep), keep), torch.where(first, keep * begin, torch.zeros_like(keep)) + take * value)
    before = torch.where(first, begin, torch.cat([h[:1], h[:-1]]))
    return h, before, keep, take, value, inside, first


def _scan(s):
    if own:
        s["call"](s["gate"], s["value"], out=s["y"], offsets=s["offsets"], sequences=s["case"]["sequences"], h0=s["h0"], h_last=s["h_last"], marks=s["marks"])
        return {"y": s["y"], "h_last": s["h_last"]}
    h, _, _, _, _, inside, _ = _states(s)
    offsets = _spans(s)[0]
    empty = (offsets[1:] == offsets[:-1])[:, None]
    h_last = torch.where(empty, s["h0"], h[(offsets[1:] - 1).clamp(min=0)])
    return {"y": torch.where(inside, h, torch.zeros_like(h)).to(s["value"].dtype), "h_last": h_last}


def _scan_back(s):
    if own:
        s["call"](s["dy"], s["gate"], s["value"], s["marks"], dgate=s["dgate"], dvalue=s["dvalue"], offsets=s["offsets"], sequences=s["case"]["sequences"],
                  dh_last=s["dh_last"], dh0=s["dh0"])
        return {"dgate": s["dgate"], "dvalue": s["dvalue"], "dh0": s["dh0"]}
    h, before, keep, take, value, inside, first = _states(s)
    offsets, owner, row = _spans(s)
    count = s["case"]["sequences"]
    last = (row == offsets[1:][owner.clamp(max=count - 1)] - 1)[:, None] & inside
    grad = s["dy"].float() + torch.where(last, s["dh_last"][owner.clamp(max=count - 1)], torch.zeros_like(keep))
    # backwards in time: g[t] = grad[t] + keep[t+1] g[t+1]
    after = torch.where(last | ~inside, torch.zeros_like(keep), torch.cat([keep[1:], keep[:1]]))
    g = _scan_rows(after.flip(0), torch.where(inside, grad, torch.zeros_like(grad)).flip(0)).flip(0)
    empty = (offsets[1:] == offsets[:-1])[:, None]
    at = offsets[:-1].clamp(max=len(row) - 1)
    return {"dgate": (g * (before - value) * keep * take).masked_fill(~inside, 0.0).to(s["gate"].dtype), "dvalue": (g * take).to(s["value"].dtype),
            "dh0": torch.where(empty, s["dh_last"], (g * keep)[at])}


def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    g = 1.0 / (1.0 + torch.exp(-z))
    return g * (1.0 + z * (1.0 - g))


def _gated(s):
    case = s["case"]
    if own:
        s["session"].forward(s["x"], s["w"], s["bias"], out=s["y"], pre=s["pre"])
        return {"y": s["y"], "pre": s["pre"]}
    w = s["w"].float()
    z = s["x"].float() @ (w if case["layout"] == "in_out" else w.t())
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(z[:, :case["n"]], case["act"]) * z[:, case["n"]:]
    return {"y": y.to(s["x"].dtype), "pre": z.to(s["x"].dtype) if case["pre"] else None}


def _gated_back(s):
    case = s["case"]
    if own:
        s["session"].backward(s["dy"], s["x"], s["w"], s["pre"], dx=s["dx"], dw=s["dw"], db=s["db"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    dy, x, w = s["dy"].float(), s["x"].float(), s["w"].float()
    gate, up = s["pre"][:, :case["n"]].float(), s["pre"][:, case["n"]:].float()
    dz = torch.cat([dy * up * _act_slope(gate, case["act"]), dy * _act(gate, case["act"])], 1)
    dx = dz @ (w.t() if case["layout"] == "in_out" else w)
    dw = x.t() @ dz if case["layout"] == "in_out" else dz.t() @ x
    return {"dx": dx.to(s["x"].dtype), "dw": dw.to(s["w"].dtype), "db": dz.sum(0)}


def work(case):
    op = case["op"]
    if op == "embed":
        cells = case["tokens"] * case["width"]
        # a word that occurs twice is read once: no more rows than the vocabulary has
        read = min(case["tokens"], case["vocab"]) * case["width"]
        return {"bytes": _ITEM[case["table"]] * read + _ITEM[case["out"]] * cells + 8 * case["tokens"], "flops": cells}
    if op == "embed_back":
        cells = case["tokens"] * case["width"]
        return {"bytes": _ITEM[case["dtype"]] * cells + _ITEM[case["grads"]] * case["vocab"] * case["width"] + 8 * case["tokens"], "flops": 2 * cells}
    if op in ("norm", "norm_back"):
        cells, item = case["rows"] * case["width"], _ITEM[case["dtype"]]
        if op == "norm":
            return {"bytes": 2 * item * cells + 8 * case["rows"] + 8 * case["width"], "flops": 8 * cells}
        return {"bytes": (3 + int(case["add"])) * item * cells + 8 * case["rows"] + 12 * case["width"], "flops": 14 * cells}
    if op in ("scan", "scan_back"):
        cells, item, ends = case["rows"] * case["width"], _ITEM[case["dtype"]], case["sequences"] * case["width"]
        marks = (case["rows"] // _MARK + case["sequences"]) * case["width"] * 4
        if op == "scan":
            return {"bytes": 3 * item * cells + 8 * ends + (marks if case["keep"] else 0), "flops": 8 * cells}
        return {"bytes": 5 * item * cells + 8 * ends + marks, "flops": 20 * cells}
    m, n, k, e = case["m"], case["n"], case["k"], _ITEM[case["dtype"]]
    if op == "gated":
        b = e * (m * k + 2 * k * n + m * n) + (8 * n if case["bias"] else 0) + (2 * e * m * n if case["pre"] else 0)
        return {"bytes": b, "flops": 4 * m * n * k}
    return {"bytes": e * (3 * m * n + 2 * m * k + 4 * k * n) + 8 * n, "flops": 8 * m * n * k}


# ------------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"embed": _exact_embed, "embed_back": _exact_embed_back, "norm": _exact_norm, "norm_back": _exact_norm_back, "scan": _exact_scan,
            "scan_back": _exact_scan_back, "gated": _exact_gated, "gated_back": _exact_gated_back}[case["op"]](s)


def _exact_embed(s):
    y = torch.zeros(s["case"]["tokens"], s["case"]["width"], dtype=torch.float64, device="cuda")
    at = (s["tokens"] != _IGNORE).nonzero()[:, 0]
    y[at] = torch.nn.functional.embedding(s["tokens"][at], s["table"]).double() * s["scale"]
    return {"y": y}


def _exact_embed_back(s):
    at = (s["tokens"] != _IGNORE).nonzero()[:, 0]
    words, order = s["tokens"][at].sort(stable=True)
    total = torch.zeros(s["case"]["vocab"], s["case"]["width"], dtype=torch.float64, device="cuda")
    total.index_put_((words,), s["dy"][at[order]].double(), accumulate=True)
    return {"dtable": total * s["scale"]}


def _exact_norm(s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, 1, correction=0)
    y = torch.nn.functional.layer_norm(x, (x.shape[1],), s["weight"].double(), s["bias"].double(), _EPS)
    return {"y": y, "mean": mean, "rstd": (var + _EPS) ** -0.5}


def _exact_norm_back(s):
    # mean and rstd are inputs of the call: the gradient's formula takes them as given
    x, dy, n = s["x"].double(), s["dy"].double(), s["x"].shape[1]
    rstd = s["rstd"].double()[:, None]
    hat = (x - s["mean"].double()[:, None]) * rstd
    g = dy * s["weight"].double()
    project = torch.stack([torch.ones_like(hat), hat], 1)                       # [rows, 2, n]
    dx = rstd * (g - (project.transpose(1, 2) @ (project @ g[:, :, None]))[:, :, 0] / n)
    return {"dx": dx if s["add"] is None else dx + s["add"].double(), "dweight": torch.einsum("rn,rn->n", dy, hat), "dbias": dy.sum(0)}


def _padded(s):
    """Row numbers of every sequence side by side, [longest, sequences], and where there is a row at all."""
    rows, count = s["case"]["rows"], s["case"]["sequences"]
    ends = s["offsets"].tolist() if s["offsets"] is not None else [i * (rows // count) for i in range(count + 1)]
    longest = max(max(b - a for a, b in zip(ends, ends[1:])), 1)
    at = torch.tensor(ends[:-1], device="cuda") + torch.arange(longest, device="cuda")[:, None]
    return at.clamp(max=rows - 1), at < torch.tensor(ends[1:], device="cuda")


def _exact_steps(s):
    """Every step's gate, value and the state before it, side by side for all sequences, and the states after the last."""
    at, there = _padded(s)
    # beyond a sequence's end the state stays as it is
    keep = torch.where(there[:, :, None], torch.sigmoid(s["gate"].double())[at], 1.0)
    value = s["value"].double()[at]
    h, before = s["h0"].double(), []
    for f, v in zip(keep, value):
        before.append(h)
        h = torch.lerp(v, h, f)
    return at, there, keep, value, before, h


def _exact_scan(s):
    at, there, _, _, before, h = _exact_steps(s)
    y = torch.zeros(s["value"].shape, dtype=torch.float64, device="cuda")
    y[at[there]] = torch.stack(before[1:] + [h])[there]
    return {"y": y, "h_last": h}


def _exact_scan_back(s):
    at, there, keep, value, before, _ = _exact_steps(s)
    dy = torch.where(there[:, :, None], s["dy"].double()[at], 0.0)
    g, grads = s["dh_last"].double(), []
    for f, d in zip(keep.flip(0), dy.flip(0)):
        grads.append(g + d)
        g = f * grads[-1]
    dh = torch.stack(grads[::-1])[there]
    take = torch.sigmoid(-s["gate"].double())[at[there]]
    dgate, dvalue = (torch.zeros(s["value"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    dgate[at[there]] = dh * (torch.stack(before)[there] - value[there]) * keep[there] * take
    dvalue[at[there]] = dh * take
    return {"dgate": dgate, "dvalue": dvalue, "dh0": g}


_EXACT_ACT = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


def _exact_gated(s):
    case = s["case"]
    w = s["w"].double() if case["layout"] == "out_in" else s["w"].double().T
    z = torch.nn.functional.linear(s["x"].double(), w, None if s["bias"] is None else s["bias"].double())
    gate, up = z.chunk(2, 1)
    return {"y": _EXACT_ACT[case["act"]](gate) * up, "pre": z if case["pre"] else None}


def _exact_gated_back(s):
    case = s["case"]
    x, w, z = (s[name].double().requires_grad_() for name in ("x", "w", "pre"))
    with torch.enable_grad():
        gate, up = z.chunk(2, 1)
        y = _EXACT_ACT[case["act"]](gate) * up
        dz, = torch.autograd.grad(y, z, s["dy"].double())
        out = torch.nn.functional.linear(x, w if case["layout"] == "out_in" else w.T)
    dx, dw = torch.autograd.grad(out, (x, w), dz)
    return {"dx": dx, "dw": dw, "db": dz.sum(0)}
