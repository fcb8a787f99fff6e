"""Plain numpy (fp64) forms of the operators at a language model's head and around its linear layers: log probabilities of
given tokens with entropy and alternatives, their gradient, 8-bit checkpoints, a linear layer's weight gradient.  Test
infrastructure only."""
import numpy as np

BLOCK = 32  # columns of a checkpoint's row that share a scale


def token_logprobs(z, tokens, scale, top):
    """Per row of ``z`` ``[n, vocab]`` (fp64): dict of logp, norm, entropy, top_index, top_logp, and the means of |d| and d^2
    (d: distance to the largest logit in units of log 2) that error bounds need.  ``tokens`` may be None."""
    n, vocab = z.shape
    out = {"logp": np.zeros(n), "norm": np.zeros((n, 2)), "entropy": np.zeros(n), "top_index": np.full((n, top), -1, np.int64),
           "top_logp": np.full((n, top), -np.inf), "d1": np.zeros(n), "d2": np.zeros(n)}
    for i in range(n):
        t = None if tokens is None else int(tokens[i])
        if t is not None and not 0 <= t < vocab:
            continue
        row = z[i].astype(np.float64)
        m = np.nan if np.isnan(row).any() else row.max()
        if m == -np.inf:
            out["norm"][i] = -np.inf, 0.0
            out["logp"][i] = -np.inf
            continue
        if not m < np.inf:
            out["norm"][i] = m, np.nan
            out["logp"][i] = out["entropy"][i] = np.nan
            out["top_logp"][i] = np.nan
            continue
        d = scale * (row - m)
        e = np.exp(d)
        s = e.sum()
        logp = d - np.log(s)
        p = e / s
        live = p > 0
        out["norm"][i] = m, np.log(s)
        out["entropy"][i] = -(p[live] * logp[live]).sum()
        if t is not None:
            out["logp"][i] = logp[t]
        far = np.minimum(-d[live], 1e30) / np.log(2.0)
        out["d1"][i], out["d2"][i] = (p[live] * far).sum(), (p[live] * far * far).sum()
        order = np.argsort(-row, kind="stable")[:top]
        order = order[row[order] > -np.inf]
        out["top_index"][i, :len(order)] = order
        out["top_logp"][i, :len(order)] = logp[order]
    return out


def token_logprobs_grad(z, tokens, norm, g, h, entropy, scale):
    """The gradient by the formula, from the given norms and entropies; ``g``, ``h`` ``[n]`` (zeros for none)."""
    n, vocab = z.shape
    out = np.zeros((n, vocab))
    for i in range(n):
        t = None if tokens is None else int(tokens[i])
        if t is not None and not 0 <= t < vocab:
            continue
        m, log_s = float(norm[i, 0]), float(norm[i, 1])
        if m == -np.inf:
            continue
        if np.isnan(log_s):
            out[i] = np.nan
            continue
        logp = scale * (z[i].astype(np.float64) - m) - log_s
        p = np.exp(logp)
        w = g[i] + h[i] * (np.where(p > 0, logp, 0.0) + (entropy[i] if entropy is not None else 0.0))
        out[i] = -p * w
        if t is not None:
            out[i, t] += g[i]
    return scale * out


def checkpoint_encode(x, tokens=None):
    """``(code, byte)`` of ``x`` ``[n, cols]``: e4m3 codes ``[n, columns rounded up to 32]`` and scale bytes ``[n, blocks]``."""
    n, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    wide = np.zeros((n, blocks * BLOCK))
    wide[:, :cols] = x
    if tokens is not None:
        wide[np.asarray(tokens) < 0] = 0.0
    wide = wide.reshape(n, blocks, BLOCK)
    bad = ~np.isfinite(wide).all(2)
    safe = np.where(bad[..., None], 0.0, wide)
    top = np.abs(safe).max(2)
    power = np.where(top > 0, np.maximum(np.frexp(top)[1] - 1 - 7, -126), -127)
    y = np.abs(safe) / np.exp2(power.astype(np.float64))[..., None]
    octave = np.maximum(np.frexp(y)[1] - 1, -6)
    grid = np.exp2(octave - 3.0)
    q = np.rint(y / grid) * grid  # rint: ties to even
    e = np.maximum(np.frexp(q)[1] - 1, -6)
    code = np.where(q >= 2.0 ** -6, (e + 7.0) * 8.0 + (q / np.exp2(e.astype(np.float64)) - 1.0) * 8.0, q * 512.0).astype(np.int64)
    code = np.where(bad[..., None], 0x7F, code | np.where(np.signbit(wide), 128, 0))
    return code.reshape(n, -1).astype(np.uint8), np.where(bad, 255, power + 127).astype(np.uint8)


def checkpoint_decode(code, byte, cols):
    """fp64 values of a checkpoint."""
    c = code.astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e > 0, np.exp2(e - 7.0) * (1 + f / 8.0), f / 8.0 * 2.0 ** -6)
    v = np.where(c & 128, -v, v)
    s = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127.0))
    return (v.reshape(*byte.shape, BLOCK) * s[..., None]).reshape(code.shape)[..., :cols]


def linear_grad(dy, x, scale):
    """One worker: the gradient ``scale * dy^T x`` and the sums of the magnitudes."""
    dy, x = dy.astype(np.float64), x.astype(np.float64)
    return scale * (dy.T @ x), abs(scale) * (np.abs(dy).T @ np.abs(x))
