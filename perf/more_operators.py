"""Performance cases of the operators at a language model's head and around its linear layers: log probabilities of given
tokens with entropy and top alternatives, their gradient into the logits, activation checkpoints in 8 bits (stored, read
back), and a linear layer's weight gradient from such a checkpoint into the workers' gradient buffers.

Every case can run in two ways: as elementary torch operations (``own = False``), or through the library's entry points
(``own = True``).  A checkpoint holds, for every row (token), e4m3 codes in blocks of 32 columns and a power of two for each
block; gradient buffers follow the library's layout: one flat fp32 buffer per worker.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 32  # columns of a checkpoint's row that share one scale


# --------------------------------------------------------------------------- #
# Cases
# --------------------------------------------------------------------------- #
def listed():
    lm = {"vocab": 33278}
    return [
        # one row of logits in fp32 with the five likeliest tokens: a step of generation, where latency counts
        {"name": "logprobs-1-top5", "op": "logprobs", **lm, "n": 1, "ld": 33278, "type": "f32", "top": 5, "given": True,
         "pad": 0.0, "masked": 0.0, "scale": 1.0},
        # the language model's training batch, 8 workers with 20 sequences of 35 tokens: the loss of each token
        {"name": "logprobs-8x700-bf16", "op": "logprobs", **lm, "n": 5600, "ld": 33278, "type": "bf16", "top": 0,
         "given": True, "pad": 0.1, "masked": 0.0, "scale": 1.0},
        # a long vocabulary of odd length: scoring at a temperature, half of the vocabulary masked, 20 alternatives
        {"name": "logprobs-2048x131071-top20", "op": "logprobs", "vocab": 131071, "n": 2048, "ld": 131072, "type": "bf16",
         "top": 20, "given": True, "pad": 0.1, "masked": 0.5, "scale": 1.25},
        # the training batch's gradient of the mean loss
        {"name": "logprobs-grad-8x700-bf16", "op": "logprobs_grad", **lm, "n": 5600, "ld": 33278, "type": "bf16",
         "out": "bf16", "mean": True, "entropy": False, "pad": 0.1, "masked": 0.0, "scale": 1.0},
        # few long rows in fp32, a weight for each token's log probability and entropy: a policy's gradient
        {"name": "logprobs-grad-64x131071-f32", "op": "logprobs_grad", "vocab": 131071, "n": 64, "ld": 131071, "type": "f32",
         "out": "f32", "mean": False, "entropy": True, "pad": 0.1, "masked": 0.5, "scale": 1.25},
        # one worker's activations of a step
        {"name": "checkpoint-store-700", "op": "store", "n": 700, "cols": 650, "ld": 650, "type": "f32", "pad": 0.0},
        # long sequences for 8 workers, in bf16, padded
        {"name": "checkpoint-store-8x16384", "op": "store", "n": 131072, "cols": 650, "ld": 656, "type": "bf16", "pad": 0.1},
        # the same read back
        {"name": "checkpoint-load-8x700", "op": "load", "n": 5600, "cols": 650, "ld": 650, "type": "f32"},
        {"name": "checkpoint-load-8x16384", "op": "load", "n": 131072, "cols": 650, "ld": 656, "type": "bf16"},
        # a recurrent layer's gate matrix from one sequence, the gradient arriving in fp32
        {"name": "linear-grad-1x35-gates", "op": "linear", "workers": 1, "n": 35, "rows": 2600, "cols": 650, "ld": 2600,
         "type": "f32", "accumulate": False, "scale": 1.0},
        # the decoder's layer from the training batch: every worker's whole 33278 x 650 gradient is written
        {"name": "linear-grad-8x700-decoder", "op": "linear", "workers": 8, "n": 700, "rows": 33278, "cols": 650,
         "ld": 33280, "type": "bf16", "accumulate": False, "scale": 1.0},
        # long sequences: micro-batches added to the gate matrix's gradient
        {"name": "linear-grad-8x16384-gates", "op": "linear", "workers": 8, "n": 16384, "rows": 2600, "cols": 650,
         "ld": 2600, "type": "bf16", "accumulate": True, "scale": 0.25},
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _padded(rng, width, to):
    return width if rng.random() < 0.5 else (width + to - 1) // to * to


def draw(rng):
    op = rng.choice(["logprobs", "logprobs_grad", "store", "load", "linear"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("logprobs", "logprobs_grad"):
        vocab = _log_uniform(rng, 50, 131071)
        most = min(65536, (60_000_000 if dtype == "f32" else 240_000_000) // vocab)
        case = {"op": op, "vocab": vocab, "n": _log_uniform(rng, 1, max(1, most)), "ld": _padded(rng, vocab, 64), "type": dtype,
                "pad": rng.choice([0.0, 0.1, 0.5]), "masked": rng.choice([0.0, 0.0, 0.5, 0.9]),
                "scale": rng.choice([1.0, 1.0, 0.7, 1.25])}
        if op == "logprobs":
            return {**case, "top": rng.choice([0, 1, 5, 20]), "given": rng.random() < 0.8}
        return {**case, "out": dtype, "mean": rng.random() < 0.5, "entropy": rng.random() < 0.5}
    if op in ("store", "load"):
        cols = _log_uniform(rng, 8, 8192)
        most = min(131072, 80_000_000 // cols)
        case = {"op": op, "n": _log_uniform(rng, 1, most), "cols": cols, "ld": _padded(rng, cols, 16), "type": dtype}
        return {**case, "pad": rng.choice([0.0, 0.1])} if op == "store" else case
    workers = rng.choice([1, 2, 4, 8])
    rows, cols = _log_uniform(rng, 50, 33278), _log_uniform(rng, 8, 2048)
    rows = min(rows, 170_000_000 // (workers * cols))
    most = int(min(16384, (1.4e11 if dtype == "f32" else 4.2e11) / (2.0 * workers * rows * cols), 4e8 / (workers * rows)))
    return {"op": op, "workers": workers, "n": _log_uniform(rng, 1, max(1, most)), "rows": rows, "cols": cols,
            "ld": _padded(rng, rows, 8), "type": dtype, "accumulate": rng.random() < 0.5, "scale": rng.choice([1.0, 0.25])}


# --------------------------------------------------------------------------- #
# Inputs
# --------------------------------------------------------------------------- #
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _context(name, rows, cols, workers):
    from paper_2010_16248_b200 import binding, workloads
    return binding.Context(workloads.make_table([(name, (rows, cols))]), workers)


def _rows(n, width, ld, dtype, fill=math.nan):
    """``[n, width]`` inside rows of ``ld`` elements; what lies between the rows is ``fill``."""
    return torch.full((n, ld), fill, dtype=dtype, device="cuda")[:, :width]


def prepare(case, seed):
    return {"logprobs": _prepare_logprobs, "logprobs_grad": _prepare_logprobs, "store": _prepare_store,
            "load": _prepare_load, "linear": _prepare_linear}[case["op"]](case, seed)


def _prepare_logprobs(case, seed):
    """A trained model's logits: spread by a few units, the token that came next well above the rest in most rows; masked
    tokens at -inf (never the given one); ids of -1 pad the batch, and padded rows hold NaN."""
    g = _gen(seed)
    v, n = case["vocab"], case["n"]
    dtype = _dtype(case["type"])
    tokens = torch.randint(0, v, (n,), generator=g, device="cuda")
    z = torch.empty(n, v, device="cuda").normal_(0, 2.0, generator=g)
    if case["masked"]:
        z.masked_fill_((torch.rand(v, generator=g, device="cuda") < case["masked"])[None, :], -math.inf)
    top = 8.0 * torch.rand(n, generator=g, device="cuda")
    z.scatter_(1, tokens[:, None], top[:, None])
    pad = torch.rand(n, generator=g, device="cuda") < case["pad"]
    tokens = torch.where(pad, -1, tokens)
    logits = _rows(n, v, case["ld"], dtype)
    logits.copy_(z)
    del z
    logits.masked_fill_(pad[:, None], math.nan)
    s = {"case": case, "logits": logits, "tokens": tokens, "scale": case["scale"]}
    f32 = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
    if own:
        s["ctx"] = _context("decoder", v, 8, 1)
    if case["op"] == "logprobs":
        s["tokens"] = tokens if case["given"] else None
        if not case["given"]:
            logits.masked_fill_(pad[:, None], 0.0)  # without given tokens every row counts
        if own:
            k = case["top"]
            s["results"] = {"logp": f32(n) if case["given"] else None, "norm": f32(n, 2), "entropy": f32(n),
                            "top_index": torch.empty(n, k, dtype=torch.int32, device="cuda") if k else None,
                            "top_logp": f32(n, k) if k else None}
        return s
    # what the forward pass left: the largest logit of a row, the logarithm of the sum relative to it, the entropy
    _, s["norm"], s["entropy"] = _statistics(logits, tokens, case["scale"])
    live = (~pad).sum().clamp(min=1)
    s["g_logp"] = -1.0 / live.float().reshape(1) if case["mean"] else torch.randn(n, generator=g, device="cuda") / n
    s["g_entropy"] = -0.01 * torch.rand(n, generator=g, device="cuda") if case["entropy"] else None
    s["dlogits"] = _rows(n, v, case["ld"], _dtype(case["out"]), 0.0)
    return s


def _activations(n, cols, g):
    """Hidden states: columns whose spread differs by up to 10^2, rows by up to 10, a few columns that stand out."""
    col = 10.0 ** (-2.0 * torch.rand(cols, generator=g, device="cuda"))
    col = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 20.0, col)
    row = 10.0 ** (torch.rand(n, 1, generator=g, device="cuda") - 0.5)
    return torch.empty(n, cols, device="cuda").normal_(generator=g).mul_(col).mul_(row)


def _prepare_store(case, seed):
    g = _gen(seed)
    n, cols = case["n"], case["cols"]
    x = _rows(n, cols, case["ld"], _dtype(case["type"]))
    x.copy_(_activations(n, cols, g))
    s = {"case": case, "x": x, "tokens": None}
    if case["pad"]:
        s["tokens"] = torch.where(torch.rand(n, generator=g, device="cuda") < case["pad"], -1, 7)
        x.masked_fill_((s["tokens"] < 0)[:, None], math.nan)
    if own:
        s["ctx"] = _context("layer", 8, cols, 1)
        s["code"], s["scale"] = s["ctx"].new_checkpoint(n, cols)
    return s


def _prepare_load(case, seed):
    n, cols = case["n"], case["cols"]
    s = {"case": case, "x": _rows(n, cols, case["ld"], _dtype(case["type"]), 0.0)}
    s["code"], s["scale"] = _quantise(_activations(n, cols, _gen(seed)), None)
    if own:
        s["ctx"] = _context("layer", 8, cols, 1)
    return s


def _prepare_linear(case, seed):
    """The layer's input as a checkpoint and the gradient of its output; a head's or a recurrent layer's gradient differs by
    orders of magnitude from token to token."""
    g = _gen(seed)
    w, n, rows, cols = (case[k] for k in ("workers", "n", "rows", "cols"))
    size = 10.0 ** (-3.0 * torch.rand(w * n, 1, generator=g, device="cuda"))
    dy = _rows(w * n, rows, case["ld"], _dtype(case["type"]))
    dy.copy_(torch.empty(w * n, rows, device="cuda").normal_(generator=g).mul_(size))
    s = {"case": case, "dy": dy.unflatten(0, (w, n)), "factor": case["scale"]}
    code, scale = _quantise(_activations(w * n, cols, g), None)
    s["code"], s["scale"] = code.unflatten(0, (w, n)), scale.unflatten(0, (w, n))
    stride = max(64, (rows * cols + 63) // 64 * 64)
    s["grads"] = torch.zeros(w, stride, device="cuda")
    if case["accumulate"]:
        s["grads"][:, :rows * cols].normal_(0, 1e-2, generator=g)
    if own:
        s["ctx"] = _context("layer", rows, cols, w)
        s["workspace"] = s["ctx"].new_linear_grad_workspace(0, n)
    return s


# --------------------------------------------------------------------------- #
# One pass
# --------------------------------------------------------------------------- #
def run(s):
    return {"logprobs": _logprobs, "logprobs_grad": _logprobs_grad, "store": _store, "load": _load,
            "linear": _linear}[s["case"]["op"]](s)


def _statistics(logits, tokens, scale):
    """(scale * (z - max), [max, log of the sum of their exponentials], entropy) of every row; a padded row counts as zeros, a
    row of -inf has max -inf, sum 1 and entropy 0."""
    z = logits.float()
    if tokens is not None:
        z = z.masked_fill((tokens < 0)[:, None], 0.0)
    top = z.amax(1)
    empty = top == -math.inf
    d = (z - torch.where(empty, 0.0, top)[:, None]) * scale
    e = d.exp()
    total = torch.where(empty, 1.0, e.sum(1))
    log_total = total.log()
    entropy = log_total - (e * torch.where(d == -math.inf, 0.0, d)).sum(1) / total
    if tokens is not None:
        pad = tokens < 0
        top, log_total, entropy = (torch.where(pad, 0.0, x) for x in (top, log_total, entropy))
    return d, torch.stack([top, log_total], 1), entropy


def _logprobs(s):
    case, logits, tokens = s["case"], s["logits"], s["tokens"]
    if own:
        r = s["results"]
        s["ctx"].acc_token_logprobs(logits, tokens, logp=r["logp"], norm=r["norm"], entropy=r["entropy"],
                                    top_index=r["top_index"], top_logp=r["top_logp"], scale=s["scale"])
        return {k: v for k, v in r.items() if v is not None}
    d, norm, entropy = _statistics(logits, tokens, s["scale"])
    out = {"norm": norm, "entropy": entropy}
    if tokens is not None:
        given = d.gather(1, tokens.clamp(min=0)[:, None])[:, 0] - norm[:, 1]
        out["logp"] = torch.where(tokens < 0, 0.0, given)
    if case["top"]:
        # larger logits first, of equal ones the lower index: one integer that holds both
        v = case["vocab"]
        bits = logits.float().add_(0.0).view(torch.int32).long()
        bits = torch.where(bits < 0, -2147483648 - bits, bits)  # increases with the logit
        key = bits * 4294967296 + (4294967295 - torch.arange(v, device=bits.device))
        del bits
        key = key.topk(case["top"], dim=1, sorted=True).values
        index = 4294967295 - (key & 4294967295)
        logp = d.gather(1, index) - norm[:, 1:]
        none = logp == -math.inf
        if tokens is not None:
            none |= (tokens < 0)[:, None]
        out["top_index"] = torch.where(none, -1, index).int()
        out["top_logp"] = torch.where(none, -math.inf, logp)
    return out


def _logprobs_grad(s):
    case, logits, tokens = s["case"], s["logits"], s["tokens"]
    if own:
        s["ctx"].acc_token_logprobs_grad(logits, tokens, s["norm"], s["dlogits"], g_logp=s["g_logp"], g_entropy=s["g_entropy"],
                                         entropy=s["entropy"] if case["entropy"] else None, scale=s["scale"])
        return s["dlogits"]
    logp = (logits.float() - s["norm"][:, :1]) * s["scale"] - s["norm"][:, 1:]
    p = logp.exp()
    g = s["g_logp"].expand(case["n"])
    dz = -g[:, None] * p
    if case["entropy"]:
        dz -= s["g_entropy"][:, None] * p * (torch.where(p == 0, 0.0, logp) + s["entropy"][:, None])
    dz.scatter_add_(1, tokens.clamp(min=0)[:, None], g[:, None])
    dz = torch.where((tokens < 0)[:, None], 0.0, dz * s["scale"])
    s["dlogits"].copy_(dz)
    return s["dlogits"]


def _quantise(x, tokens):
    """Codes ``[n, columns rounded up to 32]`` and scales ``[n, blocks]`` of a checkpoint: the largest magnitude of a block is
    brought into [128, 256) by a power of two and every value rounded to the nearest e4m3."""
    n, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    wide = torch.zeros(n, blocks * BLOCK, device=x.device)
    wide[:, :cols] = x.float()
    if tokens is not None:
        wide = torch.where((tokens < 0)[:, None], 0.0, wide)
    wide = wide.view(n, blocks, BLOCK)
    amax = wide.abs().amax(2)
    byte = torch.where(amax > 0, (torch.frexp(amax).exponent - 1 - 7 + 127).clamp(1, 254), 0)
    code = (wide * ((254 - byte) << 23).view(torch.float32)[..., None]).to(torch.float8_e4m3fn).view(n, blocks * BLOCK)
    return code, byte.to(torch.uint8).view(torch.float8_e8m0fnu)


def _store(s):
    if own:
        s["ctx"].acc_checkpoint_store(s["x"], s["code"], s["scale"], tokens=s["tokens"])
        return {"code": s["code"], "scale": s["scale"]}
    code, scale = _quantise(s["x"], s["tokens"])
    return {"code": code, "scale": scale}


def _values(code, scale, cols):
    """fp32 values of a checkpoint."""
    power = (scale.view(torch.uint8).int() << 23).view(torch.float32)  # (0 for the scale of a block of zeros)
    x = code.float().unflatten(-1, (-1, BLOCK)) * power[..., None]
    return x.flatten(-2)[..., :cols]


def _load(s):
    if own:
        s["ctx"].acc_checkpoint_load(s["code"], s["scale"], s["x"])
        return s["x"]
    s["x"].copy_(_values(s["code"], s["scale"], s["case"]["cols"]))
    return s["x"]


def _linear(s):
    case = s["case"]
    rows, cols = case["rows"], case["cols"]
    if own:
        s["ctx"].acc_linear_grad(0, s["dy"], s["code"], s["scale"], s["grads"], scale=s["factor"],
                                 accumulate=case["accumulate"], workspace=s["workspace"])
        return s["grads"]
    x = _values(s["code"], s["scale"], cols)
    total = torch.matmul(s["dy"].float().transpose(1, 2), x) * s["factor"]
    layer = s["grads"][:, :rows * cols]
    layer.copy_(layer + total.flatten(1) if case["accumulate"] else total.flatten(1))
    return s["grads"]


# --------------------------------------------------------------------------- #
# The least a pass has to move, and its result in 64 bits
# --------------------------------------------------------------------------- #
def work(case):
    n = case["n"]
    size = 2 if case["type"] == "bf16" else 4
    if case["op"] == "logprobs":
        live = n * (1 - case["pad"]) if case["given"] else n
        return {"bytes": live * case["vocab"] * size + n * (20.0 + 8.0 * case["top"]), "flops": live * case["vocab"] * 5.0}
    if case["op"] == "logprobs_grad":
        live, out = n * (1 - case["pad"]), 2 if case["out"] == "bf16" else 4
        return {"bytes": case["vocab"] * (live * size + n * out) + n * 24.0, "flops": live * case["vocab"] * 6.0}
    cols = case["cols"]
    kept = n * ((cols + BLOCK - 1) // BLOCK) * (BLOCK + 1.0)  # codes and scales
    if case["op"] == "store":
        return {"bytes": kept + n * (1 - case["pad"]) * cols * size + (8.0 * n if case["pad"] else 0.0), "flops": n * cols * 3.0}
    if case["op"] == "load":
        return {"bytes": kept + n * cols * size, "flops": n * cols * 1.0}
    w, rows = case["workers"], case["rows"]
    return {"bytes": w * (kept + n * rows * size + rows * cols * (8.0 if case["accumulate"] else 4.0)),
            "flops": 2.0 * w * n * rows * cols}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("logprobs", "logprobs_grad"):
        return _exact_logprobs(case, s)
    if case["op"] == "store":
        return _exact_store(case, s)
    x = s["code"].double() * _power(s["scale"].view(torch.uint8).long() - 127).repeat_interleave(BLOCK, -1)
    x = x[..., :case["cols"]]
    if case["op"] == "load":
        return x
    total = s["grads"].double()
    size = case["rows"] * case["cols"]
    for k in range(case["workers"]):
        product = torch.einsum("tr,tc->rc", s["dy"][k].double(), x[k]).reshape(-1) * case["scale"]
        total[k, :size] = total[k, :size] + product if case["accumulate"] else product
    return total


def _exact_logprobs(case, s):
    z = s["logits"].double()
    tokens = s["tokens"]
    n = case["n"]
    pad = torch.zeros(n, dtype=torch.bool, device="cuda") if tokens is None else tokens < 0
    z[pad] = 0.0
    logp = torch.log_softmax(z * case["scale"], 1)
    top = z.max(1).values
    if case["op"] == "logprobs":
        entropy = torch.special.entr(logp.exp()).sum(1)
        norm = torch.stack([top, torch.logsumexp(z * case["scale"], 1) - case["scale"] * top], 1)
        norm[pad], entropy[pad] = 0.0, 0.0
        out = {"norm": norm, "entropy": entropy}
        if tokens is not None:
            out["logp"] = torch.where(pad, 0.0, logp[torch.arange(n, device="cuda"), tokens.clamp(min=0)])
        if case["top"]:
            values = logp.topk(case["top"], 1).values
            values[pad] = -math.inf
            out["top_index"], out["top_logp"] = None, values
        return out
    p = logp.exp()
    one = torch.zeros_like(p)
    one[torch.arange(n, device="cuda"), tokens.clamp(min=0)] = 1.0
    weight = s["g_logp"].double().expand(n)[:, None]
    dz = weight * (one - p)
    if case["entropy"]:
        entropy = torch.special.entr(p).sum(1, keepdim=True)
        # d entropy / d logit = -p (log p + entropy), 0 where p is 0
        dz += s["g_entropy"].double()[:, None] * (torch.special.entr(p) - p * entropy)
    dz *= case["scale"]
    dz[pad] = 0.0
    return dz


def _power(exponent):
    """2^exponent in 64 bits, exactly."""
    return (exponent.long() + 1023 << 52).view(torch.float64)


def _exact_store(case, s):
    n, cols = case["n"], case["cols"]
    blocks = (cols + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(s["x"].double(), (0, blocks * BLOCK - cols)).reshape(n, blocks, BLOCK)
    if s["tokens"] is not None:
        x[s["tokens"] < 0] = 0.0
    amax = x.abs().amax(2, keepdim=True)
    power = torch.where(amax > 0, (torch.frexp(amax).exponent - 8).clamp(-126, 127), -127)
    y = x * _power(-power)
    grid = _power(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return {"code": (torch.round(y / grid) * grid).reshape(n, -1), "scale": _power(power)[..., 0]}
