"""CPU oracle of the training operators around the compression step: the AdamW update (states in 32 or in 8 bits), the
clip factor, and the embedding's lookup and gradient.  TEST INFRASTRUCTURE ONLY.

Plain numpy in fp64 from the inputs' own values; shares no code with the CUDA path.  ``layers`` is a sequence of
``(offset, rows, cols, kind)`` as in ``accordion_oracle``; buffers are flat ``[stride]`` arrays.
"""
from __future__ import annotations

import numpy as np

BLOCK = 256  # elements of a layer that share a scale of the 8-bit states
LOWEST_M, LOWEST_R = -117, -54  # smallest exponents of the scales


def coefficients(t, lr, beta1, beta2):
    """Step size and the root of the second moment's bias correction at step t >= 1."""
    return lr / (1.0 - beta1 ** t), np.sqrt(1.0 - beta2 ** t)


def clip_factor(norm2_layers, max_norm):
    norm = np.sqrt(np.sum(np.asarray(norm2_layers, np.float64)))
    if not np.isfinite(norm):
        return np.nan, norm
    return (max_norm / norm if norm > max_norm else 1.0), norm


def adamw(d, params, m, v, step, hyper, layers, factor=1.0, decay_vectors=True):
    """Returns the new (params, m, v, step); elements outside the layers keep their values."""
    if not np.isfinite(factor):
        return params.astype(np.float64), m.astype(np.float64), v.astype(np.float64), step
    lr, beta1, beta2, eps, wd = (float(h) for h in hyper)
    x, m, v = (np.array(a, np.float64) for a in (params, m, v))
    size, root = coefficients(step + 1, lr, beta1, beta2)
    with np.errstate(all="ignore"):
        for (off, rows, cols, kind) in layers:
            sl = slice(off, off + rows * cols)
            g = factor * np.asarray(d[sl], np.float64)
            m[sl] = beta1 * m[sl] + (1.0 - beta1) * g
            v[sl] = beta2 * v[sl] + (1.0 - beta2) * g * g
            decay = lr * wd if kind == 0 or decay_vectors else 0.0
            x[sl] = x[sl] - decay * x[sl] - size * m[sl] / (np.sqrt(v[sl]) / root + eps)
    return x, m, v, step + 1


# ---- states in 8 bits ------------------------------------------------------------------------------------------- #
def e4m3_values():
    """Value of each of the 256 codes: sign, four bits of exponent (bias 7), three of mantissa; 0x7f is not a number."""
    out = np.zeros(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        mag = f * 2.0 ** -9 if e == 0 else (1.0 + f / 8.0) * 2.0 ** (e - 7)
        if (c & 127) == 127:
            mag = np.nan
        out[c] = -mag if c & 128 else mag
    return out


def scale_values():
    """Value of each scale byte: powers of two, 255 is not a number."""
    out = 2.0 ** (np.arange(256, dtype=np.float64) - 127.0)
    out[255] = np.nan
    return out


def block_starts(layers):
    """(first element, length) of every block of BLOCK elements, layer after layer."""
    out = []
    for (off, rows, cols, kind) in layers:
        size = rows * cols
        out += [(off + b, min(BLOCK, size - b)) for b in range(0, size, BLOCK)]
    return out


def decode(codes, scales, layers):
    """fp64 values of 8-bit states (uint8 codes [stride], uint8 scales [blocks]); zero outside the layers."""
    val, sc = e4m3_values(), scale_values()
    out = np.zeros(codes.shape[0])
    for b, (s, n) in enumerate(block_starts(layers)):
        out[s:s + n] = val[codes[s:s + n]] * sc[scales[b]]
    return out


def random_words(seed, t, elements):
    """The 32 random bits of each element at step t."""
    def mix(x):
        x = np.asarray(x, np.uint64) & 0xFFFFFFFF
        x = x ^ (x >> np.uint64(16))
        x = (x * np.uint64(0x7FEB352D)) & np.uint64(0xFFFFFFFF)
        x = x ^ (x >> np.uint64(15))
        x = (x * np.uint64(0x846CA68B)) & np.uint64(0xFFFFFFFF)
        return x ^ (x >> np.uint64(16))
    key = mix(np.uint64((seed + 0x9E3779B9 * t) % (1 << 32)))
    return mix(key ^ (np.asarray(elements, np.uint64) & np.uint64(0xFFFFFFFF)))


def encode_block(x, rnd16, lowest, floor):
    """One block's scale byte and code bytes, and how far every rounding was from going the other way, in steps of the
    grid (a comparison with arithmetic of lower precision has to allow for the codes where this is tiny)."""
    if not np.all(np.isfinite(x)):
        return 255, np.where(floor & (x > 0), 1, 0).astype(np.uint8), np.full(x.shape, np.inf)
    top = np.max(np.abs(x))
    if top == 0.0:
        return 0, np.where(np.signbit(x), 128, 0).astype(np.uint8), np.full(x.shape, np.inf)
    power = max(int(np.frexp(top)[1]) - 1 - 7, lowest)
    y = np.abs(x) / 2.0 ** power
    octave = np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), -6.0)
    grid = 2.0 ** (octave - 3.0)
    at = y / grid + rnd16.astype(np.float64) / 65536.0
    low = np.floor(at)
    margin = np.minimum(at - low, low + 1.0 - at)
    q = low * grid
    # a grid value back into exponent and mantissa
    e = np.floor(np.log2(np.maximum(q, 2.0 ** -6)))
    normal = (e + 7.0) * 8.0 + (q / 2.0 ** e - 1.0) * 8.0
    code = np.where(q >= 2.0 ** -6, normal, q * 512.0).astype(np.int64)
    if floor:
        code = np.where((code == 0) & (x > 0), 1, code)
    return power + 127, (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8), margin


def adamw_8bit(d, params, m_code, r_code, m_scale, r_scale, step, hyper, layers, seed, factor=1.0, decay_vectors=True):
    """Returns a dict of the new values, the fp64 states before rounding and each code's margin."""
    m0, r0 = decode(m_code, m_scale, layers), decode(r_code, r_scale, layers)
    x, m, v, t = adamw(d, params, m0, r0 * r0, step, hyper, layers, factor, decay_vectors)
    out = {"params": x, "step": t, "m": m, "r": np.sqrt(v), "m_code": m_code.copy(), "r_code": r_code.copy(),
           "m_scale": m_scale.copy(), "r_scale": r_scale.copy(), "m_margin": np.full(x.shape, np.inf),
           "r_margin": np.full(x.shape, np.inf)}
    if t == step:
        return out
    for b, (s, n) in enumerate(block_starts(layers)):
        rnd = random_words(seed, t, np.arange(s, s + n))
        for name, bits, lowest in (("m", rnd & np.uint64(0xFFFF), LOWEST_M), ("r", rnd >> np.uint64(16), LOWEST_R)):
            byte, code, margin = encode_block(out[name][s:s + n], bits, lowest, name == "r")
            out[name + "_scale"][b] = byte
            out[name + "_code"][s:s + n] = code
            out[name + "_margin"][s:s + n] = margin
    return out


# ---- embedding ---------------------------------------------------------------------------------------------------- #
def embedding_lookup(table, tokens, scale):
    """scale * row of each token; zeros for tokens that name no row."""
    rows = table.shape[0]
    flat = np.asarray(tokens).reshape(-1)
    out = np.zeros((flat.shape[0], table.shape[1]))
    for i, t in enumerate(flat):
        if 0 <= t < rows:
            out[i] = scale * table[t].astype(np.float64)
    return out


def embedding_grad(tokens, dy, rows, scale):
    """One worker: (G, S, K): the gradient, and per row the sum of |scale * dy| and the number of tokens."""
    cols = dy.shape[1]
    G, S, K = np.zeros((rows, cols)), np.zeros((rows, cols)), np.zeros(rows, np.int64)
    for t, y in zip(tokens, dy):
        if 0 <= t < rows:
            G[t] += scale * y.astype(np.float64)
            S[t] += np.abs(scale * y.astype(np.float64))
            K[t] += 1
    return G, S, K
