"""Log probabilities of given tokens, entropy, alternatives and their gradient against the fp64 oracle, through the C-ABI.

Tolerances, u = 2^-24.  A distance d (in units of log 2) is a rounded difference times a rounded constant: 4 u |d| off.  The
exponential is off by 2^-22 of itself, once for its own and once for each time that the running sums change their reference:
at most once for each group of eight of a thread's share and 5 + 5 + 3 joins.  Sums of terms of one sign are off by u for each
addition on a term's way: 8 for each group of the share, and the joins.  All of it enters log S and the entropy as below; the
rounding to bf16 is half a step, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

from oracle import head_oracle as hor
from paper_2010_16248_b200 import binding, workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LN2 = np.log(2.0)


def _ctx():
    return binding.Context(wl.make_table([("decoder", (40, 8))]), 1)


def _rows(n, vocab, ld, dtype, offset=0, fill=float("nan")):
    """``[n, vocab]`` inside rows of ``ld`` elements, ``offset`` elements behind an aligned start; ``fill`` elsewhere."""
    flat = torch.full((offset + n * ld + vocab,), fill, dtype=dtype, device="cuda")
    return flat, flat[offset:offset + n * ld].view(n, ld)[:, :vocab]


def _logits(rng, n, vocab, kind):
    z = rng.normal(0, 2.0, (n, vocab))
    if kind == "peaked":
        z[np.arange(n), rng.integers(0, vocab, n)] += 30.0
    elif kind == "masked":
        z[:, rng.random(vocab) < 0.7] = -np.inf
        z[n // 2] = -np.inf
    elif kind == "lowest":  # all but a few at the type's lowest value; a row of nothing else
        keep = rng.random((n, vocab)) < 3.0 / vocab
        z = np.where(keep, z, -np.inf)
        z[n // 2] = -np.inf
    elif kind == "ties":
        z = rng.integers(-2, 3, (n, vocab)).astype(float)
    elif kind == "equal":
        z = np.broadcast_to(rng.normal(0, 1, (n, 1)), (n, vocab)).copy()
    elif kind == "rising":
        z = np.broadcast_to(np.linspace(-9, 9, vocab), (n, vocab)).copy()
    elif kind == "far":
        z = z + 5000.0 * rng.choice([-1, 1], (n, 1))
    return z


def _tokens(rng, n, vocab):
    t = rng.integers(0, vocab, n)
    return np.where(rng.random(n) < 0.2, -1 - rng.integers(0, 3, n), t) if n > 2 else t


def _outputs(n, top):
    f = lambda *s: torch.full(s, 77.0, device="cuda")  # noqa: E731
    return {"logp": f(n), "norm": f(n, 2), "entropy": f(n),
            "top_index": torch.full((n, top), 77, dtype=torch.int32, device="cuda") if top else None,
            "top_logp": f(n, top) if top else None}


def _bounds(r, scale, vocab):
    """Absolute error bounds of log S and entropy, and a function for a log p, from the oracle's means."""
    groups = vocab / 8 / 32 + 1  # of a lane's share, where it is largest
    ref, add = (groups + 13) * 2.0 ** -22 + 2.0 ** -22, (8 * groups + 13) * U
    log_s = 4 * U * r["d1"] + ref + add + 2 * U * np.abs(r["norm"][:, 1]) + 2 * U
    entropy = log_s + LN2 * (4 * U * r["d2"] + (2 * ref + 2 * add + 6 * U) * r["d1"]) + log_s * r["d1"] * LN2 + 2 * U * r["entropy"]
    far = lambda logp: log_s + 4 * U * (np.abs(logp) + np.abs(r["norm"][:, 1])) + 2 * U * np.abs(logp)  # noqa: E731
    return log_s, entropy, far


def _near(got, want, bound):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    top = float(np.finfo(np.float32).max)  # what fp32 does not reach it holds as an infinity (scale * the type's lowest value)
    want = np.where(np.abs(want) > top * (1 + U), np.copysign(np.inf, want), want)
    bound = np.broadcast_to(bound, want.shape)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    off = np.where(same, 0.0, np.abs(np.where(same, 0.0, got) - np.where(same, 0.0, want)))
    worst = np.where(same, 0.0, off / np.maximum(bound, 1e-300))
    assert np.all(worst <= 1.0), (float(np.max(worst)), int(np.argmax(worst)))


SIZES = [(1, 1, 1), (3, 2, 3), (5, 7, 7), (9, 33, 40), (2, 255, 255), (17, 1024, 1024), (4, 1025, 1025), (1, 4097, 4097),
         (3, 33278, 33278), (1, 33278, 33280), (700, 2049, 2051), (2, 131071, 131072)]
KINDS = ["plain", "peaked", "masked", "lowest", "ties", "equal", "rising", "far"]


@pytest.mark.parametrize("n,vocab,ld", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS)
def test_logprobs(n, vocab, ld, dtype, kind):
    rng = np.random.default_rng(vocab + len(kind))
    ctx, top, scale = _ctx(), [0, 1, 5, 20, 32][(n + vocab + len(kind)) % 5], [1.0, 0.7, 1.25][vocab % 3]
    flat, logits = _rows(n, vocab, ld, dtype, offset=vocab % 5)
    logits.copy_(torch.from_numpy(_logits(rng, n, vocab, kind)).to(dtype))
    if kind == "lowest":
        logits.copy_(torch.where(logits == -torch.inf, torch.finfo(dtype).min, logits))
    tokens = _tokens(rng, n, vocab)
    dev = torch.from_numpy(tokens).to([torch.int32, torch.int64][n % 2]).cuda()
    before = flat.clone()
    r = hor.token_logprobs(logits.double().cpu().numpy(), tokens, float(np.float32(scale)), top)
    out = _outputs(n, top)
    ctx.acc_token_logprobs(logits, dev, scale=scale, **out)
    log_s, entropy, far = _bounds(r, scale, vocab)
    assert np.array_equal(out["norm"][:, 0].double().cpu().numpy(), r["norm"][:, 0])
    _near(out["norm"][:, 1], r["norm"][:, 1], log_s)
    _near(out["entropy"], r["entropy"], entropy)
    _near(out["logp"], r["logp"], far(np.where(np.isfinite(r["logp"]), r["logp"], 0.0)))
    if top:
        assert np.array_equal(out["top_index"].cpu().numpy(), r["top_index"])
        t = r["top_logp"]
        for k in range(top):
            _near(out["top_logp"][:, k], t[:, k], far(np.where(np.isfinite(t[:, k]), t[:, k], 0.0)))
    assert torch.equal(before.view(torch.uint8), flat.view(torch.uint8)) and ctx.acc_device_status() == 0
    # the same bits again, and from each output alone
    for name in [k for k, v in out.items() if v is not None]:
        one = _outputs(n, top)[name]
        ctx.acc_token_logprobs(logits, dev, scale=scale, **{name: one})
        # (without the entropy the sums are the same ones)
        assert torch.equal(one.view(torch.uint8), out[name].view(torch.uint8)), name


@pytest.mark.parametrize("vocab", [900, 5000, 70000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_with_nan_infinity_and_ids_out_of_range(vocab, dtype):
    ctx, n = _ctx(), 6
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = torch.randn(n, vocab, generator=g, device="cuda").to(dtype)
    z[1, vocab - 1] = float("nan")
    z[2, 3] = float("inf")
    z[4] = float("nan")  # a padded row is not read
    tokens = torch.tensor([5, 5, 5, vocab, -3, vocab - 1], device="cuda")
    out = _outputs(n, 7)
    ctx.acc_token_logprobs(z, tokens, **out)
    assert ctx.acc_device_status() == binding.ACC_EINDEX
    ctx.acc_reset_device_status()
    assert ctx.acc_device_status() == 0
    r = hor.token_logprobs(z.double().cpu().numpy(), tokens.cpu().numpy(), 1.0, 7)
    for k in ("logp", "entropy", "top_logp"):
        got = out[k].cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(r[k])) and np.array_equal(np.isinf(got), np.isinf(r[k])), k
    assert np.isnan(out["logp"][1:3].cpu()).all() and (out["top_index"][1:5] == -1).all()
    assert (out["logp"][3:5] == 0).all() and (out["norm"][3:5] == 0).all() and (out["entropy"][3:5] == 0).all()
    dz = torch.full((n, vocab), 5.0, device="cuda")
    one = torch.ones(1, device="cuda")
    for h in (None, one):
        ctx.acc_token_logprobs_grad(z, tokens, out["norm"], dz, g_logp=one, g_entropy=h, entropy=out["entropy"])
        assert torch.isnan(dz[1:3]).all() and (dz[3:5] == 0).all() and torch.isfinite(dz[0]).all() and torch.isfinite(dz[5]).all()
    assert ctx.acc_device_status() == binding.ACC_EINDEX


def test_many_logits_above_the_bar_of_one_thread():
    """A stretch that one thread reads holds far more large logits than a list of candidates: taken one by one."""
    ctx, vocab, top = _ctx(), 200000, 32
    z = torch.zeros(1, vocab, device="cuda")
    z[0, ::7] = -torch.inf
    for v in range(40):  # thread v of each block: its groups of eight, 2048 elements apart
        at = torch.arange(8 * v, vocab, 2048, device="cuda")
        for k in range(8):
            z[0, (at + k).clamp(max=vocab - 1)] = 1.0 + torch.arange(len(at), device="cuda") % 50 + 0.01 * v
    out = _outputs(1, top)
    ctx.acc_token_logprobs(z, torch.zeros(1, dtype=torch.int64, device="cuda"), **out)
    r = hor.token_logprobs(z.double().cpu().numpy(), [0], 1.0, top)
    assert np.array_equal(out["top_index"].cpu().numpy(), r["top_index"])


@pytest.mark.parametrize("n,vocab,ld", SIZES)
@pytest.mark.parametrize("types", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                   (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("kind,which", [("plain", "g"), ("masked", "both"), ("lowest", "h"), ("far", "both"), ("peaked", "g")])
def test_gradient(n, vocab, ld, types, kind, which):
    rng = np.random.default_rng(vocab + len(kind))
    ctx, scale = _ctx(), [1.0, 0.7, 1.25][vocab % 3]
    flat, logits = _rows(n, vocab, ld, types[0], offset=vocab % 5)
    logits.copy_(torch.from_numpy(_logits(rng, n, vocab, kind)).to(types[0]))
    if kind == "lowest":
        logits.copy_(torch.where(logits == -torch.inf, torch.finfo(types[0]).min, logits))
    tokens = _tokens(rng, n, vocab)
    dev = torch.from_numpy(tokens).cuda()
    norm, entropy = torch.empty(n, 2, device="cuda"), torch.empty(n, device="cuda")
    ctx.acc_token_logprobs(logits, dev, norm=norm, entropy=entropy, scale=scale)
    one = n % 2 == 1
    g = torch.from_numpy(rng.normal(size=1 if one else n)).float().cuda() if which != "h" else None
    h = torch.from_numpy(rng.normal(size=n)).float().cuda() if which != "g" else None
    out_ld = ld if kind != "far" else ld + 3  # rows that start elsewhere take the narrow way
    out_flat, out = _rows(n, vocab, out_ld, types[1], offset=vocab % 5, fill=9.0)
    ctx.acc_token_logprobs_grad(logits, dev, norm, out, g_logp=g, g_entropy=h,
                                entropy=entropy if h is not None else None, scale=scale)
    f = lambda t: np.zeros(n) if t is None else np.broadcast_to(t.double().cpu().numpy(), n)  # noqa: E731
    s32 = float(np.float32(scale))
    nz, ent, z = norm.double().cpu().numpy(), entropy.double().cpu().numpy(), logits.double().cpu().numpy()
    want = hor.token_logprobs_grad(z, tokens, nz, f(g), f(h), ent, s32)
    # l = log2 p is off by 4 u |d| + 4 u |log2 S| + u |l|, p by ln 2 of that and the exponential's 2^-22
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(np.isfinite(z), np.clip(s32 * (z - np.where(np.isfinite(nz[:, :1]), nz[:, :1], 0.0)) / LN2, -1e4, 0), -200.0)
    l = d - nz[:, 1:] / LN2
    e_l = 4 * U * np.abs(d) + 4 * U * np.abs(nz[:, 1:] / LN2) + U * np.abs(l)
    p = np.exp2(np.maximum(l, -1000))
    w = f(g)[:, None] + f(h)[:, None] * (l * LN2 + ent[:, None])
    big = np.abs(f(g)[:, None]) + np.abs(f(h)[:, None]) * (np.abs(l) * LN2 + np.abs(ent[:, None]))
    bound = p * (np.abs(w) * (LN2 * e_l + 2.0 ** -22) + 8 * U * big + np.abs(f(h)[:, None]) * LN2 * e_l) * s32 + 2.0 ** -125 * (1 + big)
    bound = bound + np.abs(want) * (4 * U) + np.abs(want) * (2.0 ** -8 if types[1] == torch.bfloat16 else U) * (1 + 2.0 ** -6)
    rows = np.arange(n)[(tokens >= 0)]
    bound[rows, tokens[rows]] += 4 * U * np.abs(f(g)[rows]) * s32
    _near(out, want, bound)
    pads = out_flat.clone()
    start = vocab % 5
    for i in range(n):
        pads[start + i * out_ld:start + i * out_ld + vocab] = 9.0
    assert (pads == 9.0).all()
    if types[0] == types[1] and kind != "far":  # in place: the same bits
        ctx.acc_token_logprobs_grad(logits, dev, norm, logits, g_logp=g, g_entropy=h, entropy=entropy, scale=scale)
        assert torch.equal(logits, out)


def test_without_given_tokens():
    ctx = _ctx()
    z = torch.randn(5, 3000, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    out = _outputs(5, 4)
    del out["logp"]
    ctx.acc_token_logprobs(z, None, **out)
    r = hor.token_logprobs(z.double().cpu().numpy(), None, 1.0, 4)
    assert np.array_equal(out["top_index"].cpu().numpy(), r["top_index"])
    assert np.allclose(out["entropy"].cpu().numpy(), r["entropy"], rtol=1e-5)
    dz, h = torch.empty_like(z), torch.ones(1, device="cuda")
    ctx.acc_token_logprobs_grad(z, None, out["norm"], dz, g_entropy=h, entropy=out["entropy"])
    want = hor.token_logprobs_grad(z.double().cpu().numpy(), None, out["norm"].double().cpu().numpy(), np.zeros(5), np.ones(5),
                                   out["entropy"].double().cpu().numpy(), 1.0)
    assert np.allclose(dz.cpu().numpy(), want, rtol=1e-4, atol=1e-9)


def test_streams_graphs_and_empty_batches():
    """Two calls on two streams, a captured pass replayed on new logits, no rows at all."""
    ctx, n, vocab = _ctx(), 37, 9001
    g = torch.Generator(device="cuda").manual_seed(3)
    z = [torch.randn(n, vocab, generator=g, device="cuda") for _ in range(2)]
    tokens = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    want, got = [_outputs(n, 9) for _ in range(2)], [_outputs(n, 9) for _ in range(2)]
    for a, w in zip(z, want):
        ctx.acc_token_logprobs(a, tokens, **w)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for a, w, s in zip(z, got, streams):
            ctx.acc_token_logprobs(a, tokens, stream=s, **w)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(a[k], b[k]) for k in a)
    x, out, dz = z[0].clone(), _outputs(n, 9), torch.empty(n, vocab, device="cuda")
    one = torch.full((1,), -1.0 / n, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.acc_token_logprobs(x, tokens, **out)
        ctx.acc_token_logprobs_grad(x, tokens, out["norm"], dz, g_logp=one)
    for k in (1, 0, 1):
        x.copy_(z[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[k][name], out[name]) for name in out)
        ref = torch.empty_like(dz)
        ctx.acc_token_logprobs_grad(z[k], tokens, want[k]["norm"], ref, g_logp=one)
        assert torch.equal(ref, dz)
    empty = _outputs(0, 3)
    ctx.acc_token_logprobs(z[0][:0], tokens[:0], **empty)
    ctx.acc_token_logprobs_grad(z[0][:0], tokens[:0], empty["norm"], dz[:0], g_logp=one)
    assert ctx.last_launch_count() == 0


def test_rows_beyond_31_bits():
    """The last rows of logits whose offsets pass 2^31 elements."""
    ctx, vocab, n = _ctx(), 131072, 16500  # 2.16e9 elements of bf16: 4.3 GB
    z = torch.zeros(n, vocab, dtype=torch.bfloat16, device="cuda")
    z[-1, 77] = 3.0
    tokens = torch.full((n,), 77, device="cuda")
    logp = torch.empty(n, device="cuda")
    norm = torch.empty(n, 2, device="cuda")
    ctx.acc_token_logprobs(z, tokens, logp=logp, norm=norm)
    want = 3.0 - np.log(np.exp(3.0) + vocab - 1)
    assert abs(float(logp[-1]) - want) < 1e-5 and abs(float(logp[-2]) + np.log(vocab)) < 1e-5
    ctx.acc_token_logprobs_grad(z, tokens, norm, z, g_logp=torch.ones(1, device="cuda"))
    p = np.exp(want)
    assert abs(float(z[-1, 77]) - (1 - p)) <= 2.0 ** -8 and abs(float(z[-1, 78]) * (vocab - 1 + np.exp(3.0)) + 1) < 2.0 ** -7
    assert float(z[-1].float().sum().abs()) < 2.0 ** -7


def test_refusals():
    ctx, lib = _ctx(), binding.lib()
    z, t = torch.zeros(4, 50, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    good = dict(logp=f(4), norm=f(4, 2), entropy=f(4))
    for bad in (dict(logp=f(3)), dict(norm=f(4)), dict(entropy=f(5)), dict(top_logp=f(3, 2)), dict(top_logp=f(4)),
                dict(top_logp=f(4, 2), top_index=torch.zeros(4, 3, dtype=torch.int32, device="cuda")),
                dict(top_index=torch.zeros(4, 3, dtype=torch.int64, device="cuda")), dict(logp=f(4).half()), dict(logp=f(4).cpu())):
        with pytest.raises(ValueError):
            ctx.acc_token_logprobs(z, t, **{**good, **bad})
    for logits, tokens in ((z.half(), t), (z[0], t), (z.t(), t), (z.cpu(), t), (z, t[:3]), (z, t.float()), (z, t.cpu()), (z.tolist(), t)):
        with pytest.raises(ValueError):
            ctx.acc_token_logprobs(logits, tokens, **good)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(top_logp=f(4, 33))):
        with pytest.raises(binding.AccError) as e:
            ctx.acc_token_logprobs(z, t, **{**good, **kw})
        assert e.value.status == 1
    with pytest.raises(binding.AccError):
        ctx.acc_token_logprobs(z, None, **good)  # logp without tokens
    with pytest.raises(binding.AccError):
        ctx.acc_token_logprobs(z, t)  # nothing asked for
    with pytest.raises(binding.AccError):
        ctx.acc_token_logprobs(z[:1].expand(4, 50), t, **good)  # rows that overlap
    dz, one = f(4, 50), f(1)
    for kw in (dict(), dict(g_entropy=one), ):
        with pytest.raises(binding.AccError) as e:
            ctx.acc_token_logprobs_grad(z, t, good["norm"], dz, **kw)
        assert e.value.status == 1
    with pytest.raises(binding.AccError):
        ctx.acc_token_logprobs_grad(z, None, good["norm"], dz, g_logp=one)
    with pytest.raises(binding.AccError):  # in place under another type
        ctx.acc_token_logprobs_grad(z, t, good["norm"], z.view(torch.bfloat16)[:, :50], g_logp=one)
    for kw in (dict(g_logp=f(3)), dict(g_logp=one.double()), dict(g_logp=one, entropy=f(3))):
        with pytest.raises(ValueError):
            ctx.acc_token_logprobs_grad(z, t, good["norm"], dz, **kw)
    with pytest.raises(ValueError):
        ctx.acc_token_logprobs_grad(z, t, good["norm"], f(4, 49), g_logp=one)
    a, p = z.data_ptr(), good["logp"].data_ptr()
    call = lambda **k: lib.acc_token_logprobs(ctx._h, *{**dict(z=a, zt=0, n=4, v=50, ld=50, t=t.data_ptr(), tt=1, s=1.0, logp=p,  # noqa: E731
                                                               norm=None, ent=None, top=0, ti=None, tl=None), **k}.values(), None)
    assert [call(zt=2), call(tt=2), call(n=-1), call(n=(1 << 28) + 1), call(v=0), call(ld=49), call(z=None), call(top=3),
            call(top=-1)] == [1] * 9
    assert [call(z=a + 2), call(t=t.data_ptr() + 4), call(logp=p + 2), call(norm=p + 4)] == [2] * 4
    assert call(zt=1, z=a + 2) == 0 and call(n=0, z=None, t=None) == 0
