"""Log probabilities and their gradient over the range of logits and scales: masks of finite values of every size, rows far from
zero, very small and very large scales, against the fp64 oracle.  Tolerances: those of ``test_gpu_logprobs`` (a distance is off
by 4 u |d|, a sum's change of reference by 2^-22)."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as hor
from paper_2010_16248_b200 import binding
from tests.test_gpu_logprobs import _bounds, _ctx, _near, _outputs, _rows

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


def _check(z, dtype, scale, top=5, grad=True):
    """The outputs and (of a loss that is the first token's log probability and the entropy) the gradient of rows ``z``."""
    n, vocab = z.shape
    ctx = _ctx()
    _, logits = _rows(n, vocab, vocab + 3, dtype, offset=vocab % 5)
    logits.copy_(torch.from_numpy(z).to(dtype))
    exact = logits.double().cpu().numpy()
    tokens = np.array([np.argmax(exact[i]) if i % 2 else (7 * i) % vocab for i in range(n)])
    dev = torch.from_numpy(tokens).cuda()
    s32 = float(np.float32(scale))
    r = hor.token_logprobs(exact, tokens, s32, top)
    out = _outputs(n, top)
    ctx.acc_token_logprobs(logits, dev, scale=scale, **out)
    log_s, entropy, far = _bounds(r, scale, vocab)
    assert np.array_equal(out["norm"][:, 0].double().cpu().numpy(), r["norm"][:, 0])
    _near(out["norm"][:, 1], r["norm"][:, 1], log_s)
    _near(out["entropy"], r["entropy"], entropy)
    _near(out["logp"], r["logp"], far(np.where(np.isfinite(r["logp"]), r["logp"], 0.0)))
    assert np.array_equal(out["top_index"].cpu().numpy(), r["top_index"])
    for k in range(top):
        _near(out["top_logp"][:, k], r["top_logp"][:, k], far(np.where(np.isfinite(r["top_logp"][:, k]), r["top_logp"][:, k], 0.0)))
    if not grad:
        return
    g = torch.full((1,), 0.5 / s32, device="cuda")  # (so that the results keep an ordinary size)
    h = torch.full((1,), -0.25 / s32, device="cuda")
    dz = torch.empty(n, vocab, device="cuda")
    ctx.acc_token_logprobs_grad(logits, dev, out["norm"], dz, g_logp=g, g_entropy=h, entropy=out["entropy"], scale=scale)
    gs, hs = float(g) * s32, float(h) * s32
    want = hor.token_logprobs_grad(exact, tokens, r["norm"], np.full(n, gs), np.full(n, hs), r["entropy"], s32) / s32
    logp = s32 * (exact - np.where(np.isfinite(r["norm"][:, :1]), r["norm"][:, :1], 0.0)) - r["norm"][:, 1:]
    p = np.exp(np.minimum(logp, 0.0))
    live = np.where(p > 0, logp, 0.0)
    # log p: 4 u of the distance, the norm's and the entropy's own errors; p: ln 2 of the former in log 2 units, 2^-22
    e = 6 * U * (np.abs(live) + np.abs(r["norm"][:, 1:])) + log_s[:, None] + 2.0 ** -22
    big = abs(gs) + abs(hs) * (np.abs(live) + r["entropy"][:, None])
    bound = p * (big * (e + 8 * U) + abs(hs) * (e + entropy[:, None])) + 4 * U * abs(gs) * (p > 0) + 2.0 ** -120
    _near(dz, want, bound + 4 * U * np.abs(want))


def _masked(rng, n, vocab, value, where):
    z = rng.normal(0, 2.0, (n, vocab))
    if where == "70 %":
        z[rng.random((n, vocab)) < 0.7] = value
    elif where == "95 %":
        z[rng.random((n, vocab)) < 0.95] = value
    elif where == "head":
        z[:, :vocab * 2 // 3] = value
    elif where == "tail":
        z[:, vocab // 3:] = value
    else:
        z[:] = value
        z[n - 1, vocab // 2] = 1.0  # (and one row with a single logit left)
    return z


@pytest.mark.parametrize("value", [-1e9, -5e9, -1e10, -1e12, -1e18, -1e20, -1e29, -1e30])
@pytest.mark.parametrize("where", ["70 %", "95 %", "head", "tail", "all"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [900, 33278, 131071])
def test_finite_masks(value, where, dtype, vocab):
    rng = np.random.default_rng(vocab)
    _check(_masked(rng, 3, vocab, value, where), dtype, [1.0, 0.7][int(abs(value)) % 2 if abs(value) < 1e12 else 1], grad=vocab < 40000)


def test_finite_masks_of_many_rows():
    """As many rows as give each one block or one warp."""
    rng = np.random.default_rng(1)
    for n, vocab in ((400, 9000), (5000, 2000)):
        for value in (-1e10, -1e20):
            _check(_masked(rng, n, vocab, value, "70 %"), torch.bfloat16, 1.0, grad=False)


@pytest.mark.parametrize("center", [1e9, -1e9, 5e9, -5e9, 1e10, -1e10, 1e12, -1e12, 9e29, -9e29])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [900, 9000])
def test_rows_far_from_zero(center, dtype, vocab):
    rng = np.random.default_rng(vocab)
    z = center * (1 + 2.0 ** (-20 if dtype is torch.float32 else -7) * rng.integers(-8, 9, (3, vocab)))
    z[1] = center
    _check(z, dtype, 1.0)


@pytest.mark.parametrize("factor", [0.1, 0.5, 0.69, 0.6931, 0.6932, 0.7, 1.0, 4.0, 64.0, 4096.0])
@pytest.mark.parametrize("center", [300.0, -300.0, 5e9, -1e20])
@pytest.mark.parametrize("vocab", [900, 9000])
def test_rows_around_the_references_limit(factor, center, vocab):
    """Distances of ordinary size between logits whose product with the scale is 2^17 to 2^33: on both sides of the size up to
    which the kernels take distances from a rounded reference, and across it inside a row."""
    rng = np.random.default_rng(vocab)
    z = center * (1 + 2.0 ** -20 * rng.integers(-8, 9, (3, vocab)))
    _check(z, torch.float32, factor * 2.0 ** 20 / abs(center))


@pytest.mark.parametrize("scale", [1e-4, 1e-8, 1e8, 1e9, 1e10, 1e30])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [900, 9000])
def test_scales(scale, dtype, vocab):
    rng = np.random.default_rng(vocab)
    _check(rng.normal(0, 2.0, (5, vocab)), dtype, scale)


@pytest.mark.parametrize("scale", [3e-3, 2e-3, 1e-3, 1e-4, 1e-6, 1e-20, 1e-30, 1e-36, 1e-37, 1e-38])
@pytest.mark.parametrize("mask", ["-inf", "lowest", "both"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 900, 9000])
def test_masks_at_small_scales(scale, mask, dtype, vocab):
    """A logit of -inf has no share of the row whatever the scale; a finite one does where the scale leaves it one."""
    rng = np.random.default_rng(vocab)
    z = rng.normal(0, 2.0, (4, vocab))
    at = rng.random((4, vocab))
    if mask != "-inf":
        z[at < 0.3] = float(torch.finfo(dtype).min)
    if mask != "lowest":
        z[at > 0.7] = -np.inf
    z[2] = -np.inf if mask == "-inf" else float(torch.finfo(dtype).min)
    _check(z, dtype, scale)


def test_largest_scale():
    """Up to 2^127; where scale log2(e) is beyond fp32 the calls refuse."""
    rng = np.random.default_rng(7)
    for vocab in (900, 9000):
        for peak in (0.0, 3.0, -2.0 ** -100):
            z = np.minimum(rng.normal(0, 2.0, (3, vocab)), 0.0) + peak
            z[:, ::17] = peak
            _check(z, torch.float32, 2.0 ** 127)
    ctx, z, t = _ctx(), torch.zeros(2, 50, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    logp, norm, one = torch.zeros(2, device="cuda"), torch.zeros(2, 2, device="cuda"), torch.ones(1, device="cuda")
    for scale in (2.4e38, 3e38):
        with pytest.raises(binding.AccError) as e:
            ctx.acc_token_logprobs(z, t, logp=logp, scale=scale)
        assert e.value.status == 1
        with pytest.raises(binding.AccError) as e:
            ctx.acc_token_logprobs_grad(z, t, norm, z.clone(), g_logp=one, scale=scale)
        assert e.value.status == 1
