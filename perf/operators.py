"""Performance cases of the training operators around the compression step: the AdamW update over a layer table (states in
32 or in 8 bits, optionally clipped by the global gradient norm), the embedding lookup, and the embedding's gradient.

Every case can run in two ways: as elementary torch operations (``own = False``), or through the library's entry points
(``own = True``).  Buffers follow the library's layout: one flat fp32 buffer per worker, every layer at a multiple of four
elements, padding zero.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 256  # elements of a layer that share one scale of the 8-bit states
MASK32 = 0xFFFFFFFF


# --------------------------------------------------------------------------- #
# Cases
# --------------------------------------------------------------------------- #
def listed():
    lstm = {"table": "lstm", "vocab": 33278, "hidden": 650}
    resnet = {"table": "resnet18", "width": 64}
    emb = {"vocab": 33278, "hidden": 650}
    return [
        # one convolution's matrix: the smallest update, where latency counts
        {"name": "adamw-conv256x1152", "op": "adamw", "bits": 32, "table": "single", "rows": 256, "cols": 1152, "clip": False},
        # many small tensors (62 layers, 11.2 M parameters), clipped by the global norm
        {"name": "adamw-resnet18-clip", "op": "adamw", "bits": 32, **resnet, "clip": True},
        # the language model's 50.1 M parameters: bandwidth
        {"name": "adamw-lstm", "op": "adamw", "bits": 32, **lstm, "clip": False},
        # the same tables with the states in 8 bits
        {"name": "adamw8-resnet18", "op": "adamw", "bits": 8, **resnet, "clip": False},
        {"name": "adamw8-lstm-clip", "op": "adamw", "bits": 8, **lstm, "clip": True},
        # odd sizes: no row, layer or block of 256 ends on a round number
        {"name": "adamw8-odd", "op": "adamw", "bits": 8, "table": "lstm", "vocab": 5003, "hidden": 333, "clip": False},
        # one token for each of 8 sequences: generation
        {"name": "lookup-8-tokens", "op": "lookup", **emb, "workers": 8, "tokens": 1, "type": "f32", "scale": 1.0, "pad": 0.0},
        # the training batch of the language model, 20 sequences of 35 tokens for each of 8 workers
        {"name": "lookup-8x700", "op": "lookup", **emb, "workers": 8, "tokens": 700, "type": "f32", "scale": 1.0, "pad": 0.0},
        # long sequences, scaled by the square root of the width, activations in bf16, a padded batch
        {"name": "lookup-8x16384-bf16", "op": "lookup", **emb, "workers": 8, "tokens": 16384, "type": "bf16",
         "scale": 25.495097567963924, "pad": 0.1},
        # the training batch's gradient: every worker's whole 33278 x 650 layer is written, 2 % of its rows are not zero
        {"name": "grad-8x700", "op": "grad", **emb, "workers": 8, "tokens": 700, "type": "f32", "scale": 1.0, "pad": 0.0,
         "accumulate": False},
        # the same added to a gradient that is there already (weights shared with the decoder, micro-batches)
        {"name": "grad-8x700-accumulate", "op": "grad", **emb, "workers": 8, "tokens": 700, "type": "f32", "scale": 1.0,
         "pad": 0.0, "accumulate": True},
        # long sequences in bf16, padded
        {"name": "grad-8x16384-bf16", "op": "grad", **emb, "workers": 8, "tokens": 16384, "type": "bf16",
         "scale": 25.495097567963924, "pad": 0.1, "accumulate": False},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["adamw", "adamw", "lookup", "grad"])
    vocab, hidden = _log_uniform(rng, 50, 33278), _log_uniform(rng, 8, 650)
    if op == "adamw":
        case = {"op": op, "bits": rng.choice([32, 8]), "clip": rng.random() < 0.5}
        kind = rng.choice(["lstm", "resnet18", "single"])
        if kind == "lstm":
            return {**case, "table": kind, "vocab": vocab, "hidden": hidden}
        if kind == "resnet18":
            return {**case, "table": kind, "width": rng.randint(4, 64)}
        return {**case, "table": kind, "rows": _log_uniform(rng, 1, 4000), "cols": _log_uniform(rng, 1, 4000)}
    workers = rng.choice([1, 2, 3, 4, 8])
    dtype = rng.choice(["f32", "bf16"])
    most = (65536 if op == "lookup" else 32768) if dtype == "f32" else 131072
    case = {"op": op, "vocab": vocab, "hidden": hidden, "workers": workers,
            "tokens": _log_uniform(rng, 1, most // workers), "type": dtype, "scale": rng.choice([1.0, math.sqrt(hidden)]),
            "pad": rng.choice([0.0, 0.0, 0.1, 0.5])}
    if op == "grad":
        case["accumulate"] = rng.random() < 0.5
    return case


# --------------------------------------------------------------------------- #
# Layer tables
# --------------------------------------------------------------------------- #
def _shapes(case):
    if case["table"] == "single":
        return [("weight", (case["rows"], case["cols"]))]
    if case["table"] == "lstm":
        v, h = case["vocab"], case["hidden"]
        layer = [("ih", (4 * h, h)), ("hh", (4 * h, h)), ("ih.bias", (4 * h,)), ("hh.bias", (4 * h,))]
        return [("encoder", (v, h))] + layer + layer + [("decoder", (v, h)), ("decoder.bias", (v,))]
    w = case["width"]  # ResNet-18 on 32 x 32 images, convolutions as out x (in * k * k)
    convs = [(w, 27)]
    stages = [(w, w)] + [(w * m // 2, w * m) for m in (2, 4, 8)]
    for cin, cout in stages:
        convs += [(cout, 9 * cin), (cout, 9 * cout)] + ([(cout, cin)] if cin != cout else []) + [(cout, 9 * cout)] * 2
    s = []
    for n, m in convs:
        s += [("conv", (n, m)), ("bn.weight", (n,)), ("bn.bias", (n,))]
    return s + [("linear", (100, 8 * w)), ("linear.bias", (100,))]


def _layout(shapes):
    """(offset, size) of each layer and the length of the buffer."""
    sizes = np.array([int(np.prod(s)) for _, s in shapes], np.int64)
    starts = np.concatenate([[0], np.cumsum((sizes + 3) // 4 * 4)])
    return starts[:-1], sizes, max(64, int(starts[-1] + 63) // 64 * 64)


def _context(shapes, workers):
    from paper_2010_16248_b200 import binding, workloads
    return binding.Context(workloads.make_table(shapes), workers)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _expand(values, offset, sizes, stride, fill=0):
    """A buffer that holds values[l] on layer l's elements and `fill` on the padding."""
    ends = np.concatenate([offset[1:], [stride]])
    counts = torch.from_numpy(np.stack([sizes, ends - offset - sizes], 1).reshape(-1)).cuda()
    both = torch.stack([values, torch.full_like(values, fill)], 1).reshape(-1)
    return torch.repeat_interleave(both, counts)


# --------------------------------------------------------------------------- #
# Inputs
# --------------------------------------------------------------------------- #
def prepare(case, seed):
    return _prepare_adamw(case, seed) if case["op"] == "adamw" else _prepare_embedding(case, seed)


def _prepare_adamw(case, seed):
    """A run in its middle: parameters, a gradient whose scale differs between layers by up to 10^3, states that fit it, the
    step count and the hyper-parameters on the device."""
    g = _gen(seed)
    shapes = _shapes(case)
    offset, sizes, stride = _layout(shapes)
    n_layers = len(shapes)
    scale = 10.0 ** (-4.0 + 3.0 * torch.rand(n_layers, generator=g, device="cuda"))
    scale = _expand(scale, offset, sizes, stride)  # 0 on the padding
    randn = lambda: torch.randn(stride, generator=g, device="cuda")  # noqa: E731
    d = randn() * scale
    # where the gradient is row-sparse (the encoder), most elements have not moved lately: states from 1 to 10^-4 of the scale
    spread = scale * 10.0 ** (-4.0 * torch.rand(stride, generator=g, device="cuda") ** 3)
    m = randn() * spread * 0.3
    r = randn().abs_().add_(0.5) * spread
    s = {"case": case, "d": d, "params": randn() * 0.05 * (scale > 0), "step": torch.tensor([1000 + seed % 997], device="cuda"),
         "hyper": torch.tensor([1e-3, 0.9, 0.999, 1e-8, 0.01], dtype=torch.float64, device="cuda")}
    if case["clip"]:
        n2 = float((d.double() ** 2).sum())
        s["max_norm"] = 0.7 * math.sqrt(n2)  # the usual early-phase case: the clip is active
    if case["bits"] == 32:
        s["m"], s["v"] = m, r * r
    else:
        # block b of a layer: its elements [256 b, 256 b + 256)
        blocks = (sizes + BLOCK - 1) // BLOCK
        first = np.concatenate([[0], np.cumsum(blocks)])
        nb = int(first[-1])
        layer = np.repeat(np.arange(n_layers), blocks)
        start = offset[layer] + (np.arange(nb) - first[layer]) * BLOCK
        length = np.minimum(BLOCK, offset[layer] + sizes[layer] - start)
        start, length = torch.from_numpy(start).cuda(), torch.from_numpy(length).cuda()
        lane = torch.arange(BLOCK, device="cuda")
        at = start[:, None] + torch.minimum(lane[None, :], length[:, None] - 1)
        block = torch.zeros(stride, dtype=torch.int64, device="cuda")
        block[at] = torch.arange(nb, device="cuda")[:, None]
        s.update(at=at, block=block, seed=seed & 0x7FFFFFFF)
        for name, x, low in (("m", m, 10), ("r", r, 73)):
            byte = _scale_byte(x.abs()[at].amax(1), low)
            s[name + "_scale"] = byte.to(torch.uint8).view(torch.float8_e8m0fnu)
            s[name + "_code"] = (x * torch.exp2(127.0 - byte)[block]).to(torch.float8_e4m3fn)
    if own:
        s["ctx"] = _context(shapes, 1)
        s["norm2"] = torch.zeros(n_layers, dtype=torch.float64, device="cuda")
        s["factor"] = torch.zeros(1, device="cuda")
    return s


def _zipf(case):
    p = 1.0 / np.arange(1, case["vocab"] + 1)
    return p / p.sum()


def _prepare_embedding(case, seed):
    """Zipf-distributed token ids over a permutation of the rows; ids of -1 pad the batch, and the gradient at padded
    positions holds whatever an earlier kernel left there (NaN here)."""
    g = _gen(seed)
    v, h, w, n = case["vocab"], case["hidden"], case["workers"], case["tokens"]
    cdf = torch.from_numpy(np.cumsum(_zipf(case))).cuda()
    rank = torch.searchsorted(cdf, torch.rand(w, n, generator=g, device="cuda", dtype=torch.float64)).clamp_(max=v - 1)
    tokens = torch.randperm(v, generator=g, device="cuda")[rank]
    tokens = torch.where(torch.rand(w, n, generator=g, device="cuda") < case["pad"], -1, tokens)
    dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
    stride = _layout([("encoder", (v, h))])[2]
    s = {"case": case, "tokens": tokens, "scale": case["scale"]}
    if own:
        s["ctx"] = _context([("encoder", (v, h))], w)
    if case["op"] == "lookup":
        s["params"] = torch.zeros(stride, device="cuda")
        s["params"][:v * h].normal_(0, 0.1, generator=g)
        s["out"] = torch.empty(w, n, h, dtype=dtype, device="cuda")
        return s
    dy = torch.randn(w, n, h, generator=g, device="cuda") * 1e-2
    s["dy"] = torch.where((tokens < 0)[..., None], math.nan, dy).to(dtype)
    s["grads"] = torch.zeros(w, stride, device="cuda")
    if case["accumulate"]:
        s["grads"][:, :v * h].normal_(0, 1e-2, generator=g)
    if own:
        s["workspace"] = s["ctx"].new_embedding_workspace(0, n)
    return s


# --------------------------------------------------------------------------- #
# One pass
# --------------------------------------------------------------------------- #
def run(s):
    return {"adamw": _adamw, "lookup": _lookup, "grad": _grad}[s["case"]["op"]](s)


def _adamw(s):
    names = ["params", "step"] + (["m", "v"] if s["case"]["bits"] == 32 else ["m_code", "r_code", "m_scale", "r_scale"])
    if own:
        ctx, factor = s["ctx"], None
        if s["case"]["clip"]:
            factor = s["factor"]
            ctx.acc_layer_norms(s["d"], 1, s["norm2"])
            ctx.acc_clip_factor(s["norm2"], s["max_norm"], factor)
        if s["case"]["bits"] == 32:
            ctx.acc_adamw(s["d"], s["params"], s["m"], s["v"], s["step"], s["hyper"], grad_scale=factor)
        else:
            ctx.acc_adamw_8bit(s["d"], s["params"], s["m_code"], s["r_code"], s["m_scale"], s["r_scale"], s["step"],
                               s["hyper"], seed=s["seed"], grad_scale=factor)
        return {k: s[k] for k in names}
    lr, b1, b2, eps, wd = s["hyper"].unbind()
    g = s["d"]
    if s["case"]["clip"]:
        norm = (g.double() ** 2).sum().sqrt()
        g = g * torch.clamp(s["max_norm"] / norm, max=1.0).float()
    s["step"] += 1
    t = s["step"].double()[0]
    if s["case"]["bits"] == 32:
        m, v = s["m"], s["v"]
        m.mul_(b1).add_(g * (1 - b1))
        v.mul_(b2).add_(g * g * (1 - b2))
        r = v.sqrt()
    else:
        m_scale, r_scale = (s[k + "_scale"].view(torch.uint8).float().sub_(127.0).exp2_()[s["block"]] for k in ("m", "r"))
        m = s["m_code"].float() * m_scale
        r = s["r_code"].float() * r_scale
        m = m * b1 + g * (1 - b1)
        r = (r * r * b2 + g * g * (1 - b2)).sqrt()
    denom = r / (1 - b2 ** t).sqrt() + eps
    s["params"].mul_(1 - lr * wd).sub_(m / denom * (lr / (1 - b1 ** t)))
    if s["case"]["bits"] == 8:
        key = _mix((s["seed"] + 0x9E3779B9 * s["step"]) & MASK32)
        bits = _mix(key ^ torch.arange(m.numel(), device=m.device))
        for name, x, rnd, low in (("m", m, bits & 0xFFFF, 10), ("r", r, bits >> 16, 73)):
            byte = _scale_byte(x.abs()[s["at"]].amax(1), low)
            s[name + "_scale"].view(torch.uint8).copy_(byte)
            code = _round(x.abs() * torch.exp2(127.0 - byte)[s["block"]], rnd)
            code = torch.where((x > 0) & (code == 0), 1, code) if name == "r" else code
            code = torch.where(torch.signbit(x), code | 128, code)
            s[name + "_code"].view(torch.uint8).copy_(code)
    return {k: s[k] for k in names}


def _scale_byte(amax, low):
    """Exponent byte of a block's scale, 2^(byte - 127): the largest element lands in [128, 256)."""
    exponent = torch.frexp(amax)[1].float() - 1
    return torch.where(amax > 0, (exponent - 7 + 127).clamp(low, 254), 0.0)


def _mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & MASK32
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & MASK32
    return x ^ (x >> 16)


def _round(y, rnd):
    """Magnitude code of y >= 0 in e4m3: the bits below the third of the mantissa are cut after 16 random bits were added at
    the place just below it; below 2^-6 the grid is 2^-9."""
    normal = ((y.view(torch.int32) + (rnd << 4)) >> 20) - (120 << 3)
    small = (y * 512.0 + rnd.float() * 2.0 ** -16).floor().to(torch.int64)
    return torch.where(y >= 2.0 ** -6, normal, small).clamp(max=0x7E)


def _lookup(s):
    if own:
        s["ctx"].acc_embedding_lookup(0, s["params"], s["tokens"], s["out"], scale=s["scale"])
        return s["out"]
    v, h = s["case"]["vocab"], s["case"]["hidden"]
    tokens = s["tokens"]
    rows = s["params"][:v * h].view(v, h)[tokens.clamp(min=0)] * s["scale"]
    return torch.where((tokens < 0)[..., None], 0.0, rows).to(s["out"].dtype)


def _grad(s):
    if own:
        s["ctx"].acc_embedding_grad(0, s["tokens"], s["dy"], s["grads"], scale=s["scale"], accumulate=s["case"]["accumulate"],
                                    workspace=s["workspace"])
        return s["grads"]
    v, h, w, n = (s["case"][k] for k in ("vocab", "hidden", "workers", "tokens"))
    grads = s["grads"]
    if not s["case"]["accumulate"]:
        grads[:, :v * h].zero_()
    # equal tokens of a worker stand together after a stable sort; one sum for each run of them, in 64 bits
    tokens = s["tokens"].reshape(-1)
    worker = torch.arange(w, device=tokens.device).repeat_interleave(n)
    key, order = torch.sort(torch.where(tokens < 0, w * v, worker * v + tokens), stable=True)
    run_of = torch.cumsum(torch.cat([key.new_zeros(1), (key[1:] != key[:-1]).long()]), 0)
    value = torch.where((key < w * v)[:, None], s["dy"].reshape(w * n, h)[order].double(), 0.0)
    sums = torch.zeros(w * n, h, dtype=torch.float64, device=tokens.device).index_add_(0, run_of, value) * s["scale"]
    row_of = key.new_zeros(w * n).index_copy_(0, run_of, torch.where(key < w * v, key, 0))
    at = (row_of // v * grads.shape[1] + row_of % v * h)[:, None] + torch.arange(h, device=tokens.device)
    grads.view(-1).index_add_(0, at.reshape(-1), sums.float().reshape(-1))
    return grads


# --------------------------------------------------------------------------- #
# The least a pass has to move, and its result in 64 bits
# --------------------------------------------------------------------------- #
def work(case):
    if case["op"] == "adamw":
        n = int(_layout(_shapes(case))[1].sum())
        # gradient, parameters in and out, states in and out (and their scales)
        return {"bytes": n * 28.0 if case["bits"] == 32 else n * (16.0 + 4.0 / BLOCK), "flops": n * 15.0}
    v, h, w, n = (case[k] for k in ("vocab", "hidden", "workers", "tokens"))
    size = 2 if case["type"] == "bf16" else 4
    live = n * (1 - case["pad"])
    distinct = float((1 - (1 - _zipf(case)) ** live).sum())  # rows that a worker's tokens name
    if case["op"] == "lookup":
        rows = float((1 - (1 - _zipf(case)) ** (live * w)).sum())
        return {"bytes": w * n * (8.0 + h * size) + rows * h * 4.0, "flops": w * live * h}
    written = 2 * distinct * h * 4.0 if case["accumulate"] else v * h * 4.0
    return {"bytes": w * (n * 8.0 + live * h * size + written), "flops": w * live * h}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(case, s)
    v, h, w, n = (case[k] for k in ("vocab", "hidden", "workers", "tokens"))
    if case["op"] == "lookup":
        table = torch.cat([s["params"][:v * h].view(v, h).double(), torch.zeros(1, h, device="cuda", dtype=torch.float64)])
        return table[s["tokens"]] * case["scale"]  # a token of -1 takes the row of zeros at the end
    total = s["grads"].double()
    for k in range(w):
        token, dy = s["tokens"][k], s["dy"][k].double()
        live = token >= 0
        rows = torch.zeros(v, h, dtype=torch.float64, device="cuda")
        rows.index_put_((token[live],), dy[live] * case["scale"], accumulate=True)
        total[k, :v * h] += rows.reshape(-1)
    return total


def _exact_adamw(case, s):
    lr, b1, b2, eps, wd = s["hyper"].tolist()
    t = int(s["step"]) + 1
    g = s["d"].double()
    if case["clip"]:
        g = g * min(1.0, s["max_norm"] / float(torch.linalg.vector_norm(g)))
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m, v = (s[k + "_code"].double() * 2.0 ** (s[k + "_scale"].view(torch.uint8).double() - 127)[s["block"]] for k in ("m", "r"))
        v = v ** 2
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g ** 2, v, b2)
    params = s["params"].double()
    params = params - lr * (wd * params + (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)) ** 0.5 + eps))
    out = {"params": params, "step": None}
    if case["bits"] == 32:
        return {**out, "m": m, "v": v}
    # the random numbers, 32 bits for each element: the low half for m, the high half for r
    mul = lambda a, b: (a * b) % (1 << 32)  # noqa: E731

    def mixed(x):
        x = mul(x ^ (x >> 16), 0x7FEB352D)
        x = mul(x ^ (x >> 15), 0x846CA68B)
        return x ^ (x >> 16)

    key = mixed((s["seed"] + 0x9E3779B9 * t) % (1 << 32))
    bits = mixed(torch.arange(m.numel(), device="cuda") ^ key)
    for name, x, u, low in (("m", m, bits % 65536, -117), ("r", v.sqrt(), bits // 65536, -54)):
        top = torch.zeros(s["at"].shape[0], dtype=torch.float64, device="cuda")
        top.scatter_reduce_(0, s["block"], x.abs(), "amax")
        power = torch.where(top > 0, (torch.floor(torch.log2(top)) - 7).clamp(low, 127), -127)
        y = x.abs() / 2.0 ** power[s["block"]]
        grid = 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
        q = torch.floor(y / grid + u / 65536) * grid
        q = torch.where((q == 0) & (x > 0), 2.0 ** -9, q) if name == "r" else q
        out[name + "_code"] = torch.copysign(q, x)
        out[name + "_scale"] = 2.0 ** power
    return out
