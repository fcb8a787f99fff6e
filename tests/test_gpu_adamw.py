"""The AdamW update (states in 32 and in 8 bits) and the clip factor against the fp64 oracle, through the C-ABI.

Tolerances.  u = 2^-24 is the largest relative error of one fp32 rounding.  Per element, with f, d, m, v, x the fp32 inputs
and the coefficients rounded to fp32 once:
  m:  beta1 m carries 2 u (the coefficient, the product), (1 - beta1) g 3 u (coefficient, f d, product), the sum 1 u of the
      result: |error| <= 5 u (|beta1 m| + |(1 - beta1) g|).
  v:  a sum of non-negative terms with at most 6 u (coefficient, g twice, g g, product, sum): 6 u relative; the root halves
      it and rounds once: 4 u on r, 5 u are allowed; the root of the bias correction, the fma and eps: 8 u on the denominator.
  x:  step size (1 u), quotient (m's error / denominator + 8 u + the 2 ulp = 4 u of div.approx), the two fma (1 u each of
      what they give) and lr wd: 13 u on the quotient.
Second-order terms are covered by a factor of 1.01.  Values under 2^-126 add at most 2^-149 each.
"""
import numpy as np
import pytest
import torch

from oracle import training_oracle as tor
from paper_2010_16248_b200 import binding, workloads as wl
from tests import helpers as H

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = 2.0 ** -140


def _table_ragged():
    """Layers of 1 to 8193 elements, several of them ending inside a vector of four, a block of 256 or a tile of 8192."""
    return wl.make_table([("a", (1, 1)), ("v1", (3,)), ("b", (5, 51)), ("c", (16, 16)), ("v2", (257,)), ("d", (7, 13)),
                          ("e", (3, 2731)), ("f", (64, 128)), ("v3", (8191,)), ("g", (130, 190))])


def _covered(table):
    out = np.zeros(table.stride, bool)
    for _, sl in table.slices():
        out[sl] = True
    return out


def _hyper(lr=1e-2, b1=0.9, b2=0.999, eps=1e-8, wd=0.1):
    return torch.tensor([lr, b1, b2, eps, wd], dtype=torch.float64, device="cuda")


def _inputs(table, seed, padding=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = table.stride
    cover = torch.from_numpy(_covered(table)).cuda()
    scale = 10.0 ** (-5.0 * torch.rand(n, generator=g, device="cuda"))
    d, x, m = (torch.randn(n, generator=g, device="cuda") for _ in range(3))
    d, m = d * scale, m * scale * 0.3
    v = (torch.randn(n, generator=g, device="cuda") * scale) ** 2
    return [torch.where(cover, t, padding) for t in (d, x, m, v)]


def _np(t):
    return t.detach().cpu().numpy()


def _bounds(d, x, m, v, step, hyper, layers, factor, decay_vectors):
    """Oracle results and the elementwise error bounds derived above."""
    lr, b1, b2, eps, wd = hyper
    X, M, V, T = tor.adamw(d, x, m, v, step, hyper, layers, factor, decay_vectors)
    size, root = tor.coefficients(T, lr, b1, b2)
    parts = np.abs(b1 * m.astype(np.float64)) + np.abs((1 - b1) * factor * d.astype(np.float64))
    em = 1.01 * (5 * U * parts) + TINY
    ev = 1.01 * 6 * U * V + TINY
    denom = np.sqrt(V) / root + eps
    q = np.abs(M) / denom
    ex = 1.01 * U * (2 * np.abs(X) + 2 * lr * wd * np.abs(x) + 2 * np.abs(x) + size * (5 * parts / denom + 14 * q)) + TINY
    return X, M, V, T, ex, em, ev


def _check(got, want, bound, what):
    bad = ~(np.abs(got.astype(np.float64) - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} elements, first {np.flatnonzero(bad)[:4]}, off {np.abs(got - want)[bad][:4]}"


@pytest.mark.parametrize("clip,decay_vectors,step0,bf16", [(None, True, 0, False), (0.37, False, 1000, True),
                                                            (1.0, True, 2 ** 33, False)])
def test_adamw_matches_oracle(clip, decay_vectors, step0, bf16):
    table = _table_ragged()
    layers = H.layers_of(table)
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 3, padding=float("nan"))
    if step0 == 0:
        m.mul_(0), v.mul_(0)
    step = torch.tensor([step0], device="cuda")
    hyper = _hyper()
    factor = None if clip is None else torch.tensor([clip], device="cuda")
    low = torch.full((table.stride,), 7.0, dtype=torch.bfloat16, device="cuda") if bf16 else None
    cover = _covered(table)
    for k in range(3):
        before = [_np(t).copy() for t in (d, x, m, v)]
        f = 1.0 if clip is None else float(np.float32(clip))
        X, M, V, T, ex, em, ev = _bounds(*before, step0 + k, _np(hyper), layers, f, decay_vectors)
        ctx.acc_adamw(d, x, m, v, step, hyper, grad_scale=factor, params_bf16=low,
                      flags=0 if decay_vectors else binding.ACC_ADAMW_NO_VECTOR_DECAY)
        assert ctx.last_launch_count() == 1
        for got, want, bound, what in ((x, X, ex, "x"), (m, M, em, "m"), (v, V, ev, "v")):
            _check(_np(got)[cover], want[cover], bound[cover], what)
            assert np.isnan(_np(got)[~cover]).all()  # padding is left alone
        assert int(step) == T == step0 + k + 1
        if bf16:
            c = torch.from_numpy(cover).cuda()
            assert torch.equal(low[c], x.to(torch.bfloat16)[c]) and bool((low[~c] == 7.0).all())
        d = d.roll(8) * 0.5 if k == 0 else d
        d = torch.where(torch.from_numpy(cover).cuda(), torch.nan_to_num(d), float("nan"))


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 255, 256, 257, 1023, 1025, 2047, 2049, 8191, 8192, 8193, 20011])
def test_adamw_both_widths_at_edge_sizes(n):
    """One VECTOR layer of n elements in the middle of the buffer; nothing around it moves."""
    table = wl.make_table([("before", (5,)), ("x", (n,)), ("after", (7,))])
    sub = wl.LayerTable(["x"], table.offset[1:2], table.rows[1:2], table.cols[1:2], table.kind[1:2], table.stride)
    layers = H.layers_of(sub)
    ctx = binding.Context(sub, 1)
    assert ctx.adamw_blocks == (n + 255) // 256
    d, x, m, v = _inputs(sub, n, padding=float("nan"))
    hyper = _hyper()
    cover = _covered(sub)
    before = [_np(t).copy() for t in (d, x, m, v)]
    X, M, V, T, ex, em, ev = _bounds(*before, 4, _np(hyper), layers, 1.0, True)
    step = torch.tensor([4], device="cuda")
    xx, mm, vv = x.clone(), m.clone(), v.clone()
    ctx.acc_adamw(d, xx, mm, vv, step, hyper)
    for got, want, bound, what in ((xx, X, ex, "x"), (mm, M, em, "m"), (vv, V, ev, "v")):
        _check(_np(got)[cover], want[cover], bound[cover], what)
        assert np.isnan(_np(got)[~cover]).all()
    _check_8bit(sub, ctx, d, x, m, v, 4, hyper, seed=n)


def _pack(table, ctx, m, v):
    """8-bit states near (m, v): the codes of a rounding with fixed random words (any valid state will do)."""
    layers = H.layers_of(table)
    out = [np.full(table.stride, 0x5A, np.uint8) for _ in range(2)] + [np.zeros(ctx.adamw_blocks, np.uint8) for _ in range(2)]
    for b, (s, n) in enumerate(tor.block_starts(layers)):
        half = np.full(n, 32768)
        out[2][b], out[0][s:s + n], _ = tor.encode_block(_np(m)[s:s + n].astype(np.float64), half, tor.LOWEST_M, False)
        out[3][b], out[1][s:s + n], _ = tor.encode_block(np.sqrt(_np(v)[s:s + n].astype(np.float64)), half, tor.LOWEST_R, True)
    types = [torch.float8_e4m3fn] * 2 + [torch.float8_e8m0fnu] * 2
    return [torch.from_numpy(a).cuda().view(t) for a, t in zip(out, types)]


def _bytes(t):
    return _np(t.view(torch.uint8))


def _check_8bit(table, ctx, d, x, m, v, step0, hyper, seed, clip=None, flags=0, bf16=False, steps=2):
    layers = H.layers_of(table)
    cover = _covered(table)
    state = _pack(table, ctx, m, v)
    x = x.clone()
    step = torch.tensor([step0], device="cuda")
    factor = None if clip is None else torch.tensor([clip], device="cuda")
    low = torch.full((table.stride,), 7.0, dtype=torch.bfloat16, device="cuda") if bf16 else None
    f = 1.0 if clip is None else float(np.float32(clip))
    h = _np(hyper)
    for k in range(steps):
        b = [_bytes(t).copy() for t in state]
        x0, dh = _np(x).copy(), _np(d)
        want = tor.adamw_8bit(dh, x0, *b, step0 + k, h, layers, seed, f, not flags)
        m0, r0 = tor.decode(b[0], b[2], layers), tor.decode(b[1], b[3], layers)
        X, M, V, T, ex, em, ev = _bounds(dh, x0, m0, r0 * r0, step0 + k, h, layers, f, not flags)
        ctx.acc_adamw_8bit(d, x, *state, step, hyper, seed=seed, grad_scale=factor, params_bf16=low, flags=flags)
        assert ctx.last_launch_count() == 1 and int(step) == T
        # r r is exact (four bits squared), so x has the 32-bit update's bound
        _check(_np(x)[cover], X[cover], ex[cover], "x")
        assert np.array_equal(_np(x)[~cover], x0[~cover], equal_nan=True)
        if bf16:
            c = torch.from_numpy(cover).cuda()
            assert torch.equal(low[c], x.to(torch.bfloat16)[c]) and bool((low[~c] == 7.0).all())
        got = [_bytes(t) for t in state]
        for name, code, scale, err in (("m", got[0], got[2], em), ("r", got[1], got[3], 5.05 * U * np.sqrt(V) + TINY)):
            # (5 u on r: half of v's 6 u, the root's rounding, 1 u to spare)
            assert np.array_equal(scale, want[name + "_scale"]), name
            assert np.array_equal(code[~cover], b[0 if name == "m" else 1][~cover])
            for blk, (s, n) in enumerate(tor.block_starts(layers)):
                sl = slice(s, s + n)
                differ = code[sl] != want[name + "_code"][sl]
                if not differ.any():
                    continue
                # a code may go the other way only where the fp32 value's error, in steps of the grid, and the rounding of
                # y 512 + u (at most 8, so 2^-21) reach the threshold
                y = np.abs(want[name][sl]) / 2.0 ** (float(scale[blk]) - 127)
                grid = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), -6) - 3) * 2.0 ** (float(scale[blk]) - 127)
                reach = 1.01 * err[sl] / grid + 2.0 ** -21
                assert (want[name + "_margin"][sl][differ] <= reach[differ]).all(), name
                a, w = (tor.e4m3_values()[c[sl]][differ] for c in (code, want[name + "_code"]))
                assert (np.abs(a - w) <= grid[differ] / 2.0 ** (float(scale[blk]) - 127) * 2).all()


@pytest.mark.parametrize("clip,flags,step0,bf16", [(None, 0, 0, False), (0.37, binding.ACC_ADAMW_NO_VECTOR_DECAY, 1000, True)])
def test_adamw_8bit_matches_oracle(clip, flags, step0, bf16):
    table = _table_ragged()
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 11, padding=float("nan"))
    if step0 == 0:
        m.mul_(0), v.mul_(0)
    _check_8bit(table, ctx, d, x, torch.nan_to_num(m), torch.nan_to_num(v), step0, _hyper(), 12345, clip, flags, bf16, 3)


def test_adamw_8bit_from_fresh_states_and_layout():
    table = _table_ragged()
    ctx = binding.Context(table, 1)
    layers = H.layers_of(table)
    blocks = [(r * c + 255) // 256 for (_, r, c, _) in layers]
    assert list(ctx.adamw_block0) == list(np.cumsum([0] + blocks[:-1])) and ctx.adamw_blocks == sum(blocks)
    state = ctx.new_adamw_8bit()
    assert all(int(t.view(torch.uint8).sum()) == 0 for t in state)
    d, x, _, _ = _inputs(table, 5)
    x0 = _np(x).copy()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    ctx.acc_adamw_8bit(d, x, *state, step, _hyper(), seed=1)
    X, _, _, T, ex, _, _ = _bounds(_np(d), x0, np.zeros(table.stride), np.zeros(table.stride), 0, _np(_hyper()), layers, 1.0, True)
    cover = _covered(table)
    _check(_np(x)[cover], X[cover], ex[cover], "x")


def test_a_factor_that_is_not_finite_changes_nothing():
    table = _table_ragged()
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 7)
    d[3] = float("inf")  # padding behind the first layer's single element: not part of the norm
    n2 = torch.zeros(table.n_layers, dtype=torch.float64, device="cuda")
    factor, norm = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    ctx.acc_layer_norms(d, 1, n2)
    ctx.acc_clip_factor(n2, 1.0, factor, norm)
    assert torch.isfinite(factor).item() and torch.isfinite(norm).item()
    d[5] = float("inf")
    ctx.acc_layer_norms(d, 1, n2)
    ctx.acc_clip_factor(n2, 1.0, factor, norm)
    state = _pack(table, ctx, m, v)
    step = torch.tensor([9], device="cuda")
    for bad in (factor, torch.tensor([float("inf")], device="cuda")):
        before = [t.clone() for t in (x, m, v, step)] + [t.view(torch.uint8).clone() for t in state]
        ctx.acc_adamw(d, x, m, v, step, _hyper(), grad_scale=bad)
        ctx.acc_adamw_8bit(d, x, *state, step, _hyper(), grad_scale=bad)
        after = [x, m, v, step] + [t.view(torch.uint8) for t in state]
        assert all(torch.equal(a, b) for a, b in zip(before, after))
    assert torch.isnan(factor).item() and torch.isinf(norm).item()


def test_elements_that_are_not_finite_follow_the_formulas():
    """Without a factor: in 32 bits the element alone turns into NaN; in 8 bits its block of states does, the parameters of
    the others one step later."""
    table = wl.make_table([("a", (4, 200))])
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 1)
    d[300] = float("nan")
    step = torch.tensor([3], device="cuda")
    x1, m1, v1 = x.clone(), m.clone(), v.clone()
    ctx.acc_adamw(d, x1, m1, v1, step, _hyper())
    for t in (x1, m1, v1):
        assert torch.isnan(t).nonzero().flatten().tolist() == [300]
    state = _pack(table, ctx, m, v)
    x8 = x.clone()
    ctx.acc_adamw_8bit(d, x8, *state, step, _hyper())
    assert torch.isnan(x8).nonzero().flatten().tolist() == [300]
    assert _bytes(state[2]).tolist()[1] == 255 and _bytes(state[3]).tolist()[1] == 255
    assert all(b != 255 for s in state[2:] for b in _bytes(s)[[0, 2, 3]])
    d[300] = 0.0
    ctx.acc_adamw_8bit(d, x8, *state, step, _hyper())
    assert torch.isnan(x8).nonzero().flatten().tolist() == list(range(256, 512))


@pytest.mark.parametrize("magnitude", [1e-37, 1e-25, 1e-12, 1e12, 1e18])
def test_extreme_magnitudes(magnitude):
    """Gradients near either end of fp32: squares that underflow to 0, and squares just below overflow."""
    table = wl.make_table([("a", (3, 300)), ("b", (100,))])
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 2)
    d, m = d * magnitude, m * 0
    v = v * 0
    hyper = _hyper(eps=1e-30)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    X, M, V, T = tor.adamw(_np(d), _np(x), _np(m), _np(v), 0, _np(hyper), H.layers_of(table))
    state = ctx.new_adamw_8bit()
    x8 = x.clone()
    ctx.acc_adamw(d, x, m, v, step.clone(), hyper)
    ctx.acc_adamw_8bit(d, x8, *state, step, hyper)
    assert torch.isfinite(x).all() and torch.isfinite(m).all() and torch.isfinite(v).all()
    # m, x: where g^2 does not underflow the formulas hold; below that the denominator is eps or sqrt of a subnormal
    np.testing.assert_allclose(_np(m), M, rtol=6 * U, atol=TINY)
    if magnitude >= 1e-12:
        np.testing.assert_allclose(_np(v), V, rtol=8 * U, atol=2.0 ** -125)
        np.testing.assert_allclose(_np(x8), _np(x), rtol=0, atol=0)
    for s, low in zip(state[2:], (10, 73)):
        b = _bytes(s)
        assert ((b >= low) & (b < 255)).all() or magnitude < 1e-20
    for s in state[:2]:
        assert ((_bytes(s) & 127) != 127).all()


def test_both_widths_are_reproducible_and_streams_and_graphs_give_the_same_bits():
    table = wl.make_table(wl.shapes_resnet18(10, 16))
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 21)
    hyper = _hyper()

    def fresh():
        return [x.clone(), m.clone(), v.clone()], _pack(table, ctx, m, v), torch.tensor([5], device="cuda")

    def steps(f32, f8, s32, s8, n, stream=None):
        for _ in range(n):
            ctx.acc_adamw(d, *f32, s32, hyper, stream=stream)
            ctx.acc_adamw_8bit(d, f32[0], *f8, s8, hyper, seed=3, stream=stream)

    a32, a8, sa = fresh()
    sa8 = sa.clone()
    steps(a32, a8, sa, sa8, 4)
    b32, b8, sb = fresh()
    sb8 = sb.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    steps(b32, b8, sb, sb8, 4, stream=side)
    side.synchronize()
    c32, c8, sc = fresh()
    sc8 = sc.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(c32, c8, sc, sc8, 2)
    assert int(sc) == 5  # capturing runs nothing
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for o32, o8, s, s8 in ((b32, b8, sb, sb8), (c32, c8, sc, sc8)):
        assert int(s) == int(s8) == 9
        assert all(torch.equal(p, q) for p, q in zip(a32, o32))
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a8, o8))
    hyper[0] = 0.0  # a replayed graph follows the hyper-parameters: lr = 0 leaves the parameters
    x_now = c32[0].clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x_now, c32[0]) and int(sc) == 11


def test_8bit_second_moment_follows_a_stationary_gradient():
    """Rounding up or down at random moves the mean as the formula says.  A step moves r by |dr| ~ (1 - beta2)/2 |g^2/v - 1| r,
    0.97 (1 - beta2)/2 r on average, on a grid no coarser than r/8: the rounding's variance is at most 0.061 (1 - beta2) r^2
    a step, which the decay of v by (1 - beta2) turns into a mean of v at most 6.1 % too large (and none too small);
    65536 elements of correlation length 1/(1 - beta2) leave a sampling error of the mean below 0.1 %.
    Started at 3 times the true r, where rounding to nearest would stay for good."""
    n = 65536
    table = wl.make_table([("a", (256, 256))])
    ctx = binding.Context(table, 1)
    g = torch.Generator(device="cuda").manual_seed(4)
    beta2 = 0.99
    hyper = _hyper(lr=0.0, b2=beta2)
    x = torch.zeros(table.stride, device="cuda")
    state = _pack(table, ctx, x, torch.full_like(x, 9.0))
    step = torch.tensor([10 ** 6], device="cuda")
    for _ in range(1200):  # 12 time constants
        d = torch.randn(table.stride, generator=g, device="cuda")
        ctx.acc_adamw_8bit(d, x, *state, step, hyper, seed=9)
    r = tor.decode(_bytes(state[1]), _bytes(state[3]), H.layers_of(table))[:n]
    assert 0.99 < np.mean(r * r) < 1.07


def test_adamw_refuses_misaligned_and_missing_buffers():
    table = wl.make_table([("a", (6, 10)), ("v", (5,))])
    ctx = binding.Context(table, 1)
    S = table.stride
    big = torch.zeros(S + 4, device="cuda")
    step, hyper = torch.zeros(1, dtype=torch.int64, device="cuda"), _hyper()
    z = [torch.zeros(S, device="cuda") for _ in range(4)]
    for k in range(4):
        args = list(z)
        args[k] = big[1:S + 1]
        with pytest.raises(binding.AccError) as e:
            ctx.acc_adamw(*args, step, hyper)
        assert e.value.status == 2
    with pytest.raises(binding.AccError) as e:
        ctx.acc_adamw(*z, step, hyper, flags=2)
    assert e.value.status == 1
    state = ctx.new_adamw_8bit()
    wide = torch.zeros(S + 4, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    with pytest.raises(binding.AccError) as e:
        ctx.acc_adamw_8bit(z[0], z[1], wide[1:S + 1], *state[1:], step, hyper)
    assert e.value.status == 2
    n2, f = torch.zeros(table.n_layers, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    for bad in (-1.0, float("nan")):
        with pytest.raises(binding.AccError) as e:
            ctx.acc_clip_factor(n2, bad, f)
        assert e.value.status == 1
    lib = binding.lib()
    p = z[0].data_ptr()
    assert lib.acc_adamw(ctx._h, p, p, None, p, step.data_ptr(), hyper.data_ptr(), None, None, 0, None) == 1
    assert lib.acc_adamw(ctx._h, p, p, p, p, step.data_ptr() + 4, hyper.data_ptr(), None, None, 0, None) == 2
    assert int(step) == 0


@pytest.mark.parametrize("n_layers", [1, 2, 300, 1000])
def test_clip_factor_matches_oracle(n_layers):
    """fp64 sums of at most 1000 terms (relative error under 1000 * 2^-53), one fp32 rounding of the factor."""
    table = wl.make_table([(f"v{i}", (4,)) for i in range(n_layers)])
    ctx = binding.Context(table, 1)
    n2 = torch.rand(n_layers, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    f, norm = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    for share in (0.0, 0.3, 1.5):
        total = float(np.sqrt(_np(n2).sum()))
        want, wn = tor.clip_factor(_np(n2), share * total)
        ctx.acc_clip_factor(n2, share * total, f, norm)
        assert abs(float(f) - want) <= 1.01 * U * want and abs(float(norm) - wn) <= 1e-12 * wn
    ctx.acc_clip_factor(n2 * 0, 0.0, f)
    assert float(f) == 1.0


def test_large_tables_take_their_coefficients_from_a_kernel_ahead():
    """More blocks than fit the GPU at once: two launches, the same results; a factor that is not finite leaves everything."""
    table = wl.make_table([("a", (700, 3001)), ("v", (5003,)), ("b", (513, 1025))])
    layers, cover = H.layers_of(table), _covered(table)
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 31, padding=float("nan"))
    step, hyper = torch.tensor([17], device="cuda"), _hyper()
    factor = torch.tensor([0.25], device="cuda")
    before = [_np(t).copy() for t in (d, x, m, v)]
    X, M, V, T, ex, em, ev = _bounds(*before, 17, _np(hyper), layers, 0.25, True)
    x8, state, step8 = x.clone(), _pack(table, ctx, torch.nan_to_num(m), torch.nan_to_num(v)), step.clone()
    ctx.acc_adamw(d, x, m, v, step, hyper, grad_scale=factor)
    assert ctx.last_launch_count() == 2 and int(step) == 18
    for got, want, bound, what in ((x, X, ex, "x"), (m, M, em, "m"), (v, V, ev, "v")):
        _check(_np(got)[cover], want[cover], bound[cover], what)
        assert np.isnan(_np(got)[~cover]).all()
    b = [_bytes(t).copy() for t in state]
    want = tor.adamw_8bit(before[0], before[1], *b, 17, _np(hyper), layers, 3, 0.25)
    m0, r0 = tor.decode(b[0], b[2], layers), tor.decode(b[1], b[3], layers)
    X, M, V, T, ex, em, ev = _bounds(before[0], before[1], m0, r0 * r0, 17, _np(hyper), layers, 0.25, True)
    ctx.acc_adamw_8bit(d, x8, *state, step8, hyper, seed=3, grad_scale=factor)
    assert ctx.last_launch_count() == 2 and int(step8) == 18
    _check(_np(x8)[cover], X[cover], ex[cover], "x")
    for k, name in enumerate(("m_code", "r_code", "m_scale", "r_scale")):
        # (the codes at rounding thresholds, about one in 10^5, are examined one by one in the tests above)
        assert np.mean(_bytes(state[k]) != want[name]) < 1e-4
    factor.fill_(float("nan"))
    kept = [t.clone() for t in (x, m, v, step, x8, step8)] + [t.view(torch.uint8).clone() for t in state]
    ctx.acc_adamw(d, x, m, v, step, hyper, grad_scale=factor)
    ctx.acc_adamw_8bit(d, x8, *state, step8, hyper, seed=3, grad_scale=factor)
    now = [x, m, v, step, x8, step8] + [t.view(torch.uint8) for t in state]
    assert all(torch.equal(a.nan_to_num(7), b.nan_to_num(7)) for a, b in zip(kept, now))


def test_one_and_two_launches_give_the_same_bits():
    """The layer of a table that fits at once, alone and beside a large one."""
    shapes = [("a", (300, 700)), ("b", (2000, 2000))]
    big = wl.make_table(shapes)
    small = wl.LayerTable(["a"], big.offset[:1], big.rows[:1], big.cols[:1], big.kind[:1], big.stride)
    d, x, m, v = _inputs(big, 2)
    sl = slice(0, 210000)
    got = []
    for table in (small, big):
        ctx = binding.Context(table, 1)
        f32, f8, s, s8 = [t.clone() for t in (x, m, v)], _pack(table, ctx, m, v), torch.tensor([3], device="cuda"), torch.tensor([3], device="cuda")
        for _ in range(2):
            ctx.acc_adamw(d, *f32, s, _hyper())
            one = ctx.last_launch_count()
            ctx.acc_adamw_8bit(d, f32[0], *f8, s8, _hyper(), seed=1)
        got.append((one, [t[sl] for t in f32], [t.view(torch.uint8)[sl] for t in f8[:2]]))
    assert got[0][0] == 1 and got[1][0] == 2
    assert all(torch.equal(p, q) for k in (1, 2) for p, q in zip(got[0][k], got[1][k]))


def test_offsets_beyond_32_bits():
    """A layer behind element 2^31 + 2^20 of buffers of 8.6 GB, of which only its neighbourhood is touched."""
    off, n = 2 ** 31 + 2 ** 20, 70001
    stride = off + 70016
    table = wl.LayerTable(["far"], np.array([off], np.int64), np.array([1], np.int32), np.array([n], np.int32),
                          np.array([wl.VECTOR], np.int32), stride)
    near = wl.make_table([("near", (n,))])
    ctx, ref = binding.Context(table, 1), binding.Context(near, 1)
    small = _inputs(near, 8)
    big = [torch.empty(stride, device="cuda") for _ in range(4)]
    for b, s in zip(big, small):
        b[off:off + 70016].fill_(7.0)
        b[off:off + n] = s[:n]
    step = [torch.tensor([3], device="cuda") for _ in range(4)]
    hyper = _hyper()
    ctx.acc_adamw(*big, step[0], hyper)
    ref.acc_adamw(*small, step[1], hyper)
    for b, s in zip(big, small):
        assert torch.equal(b[off:off + n], s[:n]) and bool((b[off + n:] == 7.0).all())
    codes = [torch.zeros(stride, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(ctx.adamw_blocks, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2)]
    x0 = _np(big[1][off:off + n]).copy()
    ctx.acc_adamw_8bit(big[0], big[1], *codes, *scales, step[2], hyper, seed=5)
    rnd = tor.random_words(5, 4, np.arange(off, off + n, dtype=np.uint64))
    z = np.zeros(n)
    X, M, V, _ = tor.adamw(_np(small[0])[:n], x0, z, z, 3, _np(hyper), [(0, 1, n, 1)])
    _check(_np(big[1][off:off + n]), X, _bounds(_np(small[0])[:n], x0, z, z, 3, _np(hyper), [(0, 1, n, 1)], 1.0, True)[4], "x")
    byte, code, margin = tor.encode_block(M[:256], rnd[:256] & np.uint64(0xFFFF), tor.LOWEST_M, False)
    assert _bytes(scales[0])[0] == byte and np.mean(_np(codes[0].view(torch.uint8)[off:off + 256]) != code) < 0.02
    assert int(codes[0].view(torch.uint8)[:off].count_nonzero()) == 0


@pytest.mark.parametrize("power", [-30, 0, 20])
@pytest.mark.parametrize("which", ["m", "r"])
def test_adamw_8bit_codes_next_to_a_carry(which, power):
    """Codes below the normal ones, 2^-22 of a step under the value from which their random bits would carry them to the
    next: rounding the scaled value to the 2^-20 of a step that are kept would carry them all.  beta1 = 1/2 and beta2 = 3/4
    make m = g / 2 and r = |g| / 2 exact, so a gradient puts any value there."""
    n, t, seed = 256 * 64, 8, 11
    table = wl.make_table([("x", (n,))])
    ctx = binding.Context(table, 1)
    u = tor.random_words(seed, t, np.arange(n))
    u = (u & np.uint64(0xFFFF) if which == "m" else u >> np.uint64(16)).astype(np.float64)
    y = (1.0 + (65536.0 - u) / 65536.0 - 2.0 ** -22) / 512.0  # code 1, its random bits just short of code 2
    y[::256] = 128.0  # a block's largest element: the scale is 2^power
    y[3::7] *= -1.0
    d = torch.zeros(table.stride, device="cuda")
    exact = 2.0 * y * 2.0 ** power
    d[:n] = torch.from_numpy(exact.astype(np.float32)).cuda()
    assert np.array_equal(_np(d[:n]).astype(np.float64), exact)
    state, x = ctx.new_adamw_8bit(), torch.zeros(table.stride, device="cuda")
    ctx.acc_adamw_8bit(d, x, *state, torch.tensor([t - 1], device="cuda"), _hyper(b1=0.5, b2=0.75), seed=seed)
    code, scale = (_bytes(state[k]) for k in ((0, 2) if which == "m" else (1, 3)))
    assert (scale == 127 + power).all()
    small = np.abs(y) < 1.0
    sign = np.where((y < 0) & (which == "m"), 128, 0)
    assert np.array_equal(code[:n][small], (1 | sign)[small])


def _codes_by_fp32(d, b, step0, hyper, layers, seed, f):
    """The 8-bit states after a step, from the formulas taken operation by operation in fp32 and the codes' rounding in fp64,
    which is exact for fp32 values."""
    lr, b1, b2, eps, wd = hyper
    one = np.float32
    val, sc = tor.e4m3_values().astype(one), tor.scale_values().astype(one)
    out = [a.copy() for a in b]
    for k, (s, n) in enumerate(tor.block_starts(layers)):
        sl = slice(s, s + n)
        g = one(f) * d[sl]
        m = (sc[b[2][k]] * one(b1)) * val[b[0][sl]] + one(1.0 - b1) * g
        r = val[b[1][sl]]
        v = (sc[b[3][k]] * sc[b[3][k]] * one(b2)) * (r * r) + one(1.0 - b2) * (g * g)
        assert m.dtype == v.dtype == one
        rnd = tor.random_words(seed, step0 + 1, np.arange(s, s + n))
        out[2][k], out[0][sl], _ = tor.encode_block(m.astype(np.float64), rnd & np.uint64(0xFFFF), tor.LOWEST_M, False)
        out[3][k], out[1][sl], _ = tor.encode_block(np.sqrt(v).astype(np.float64), rnd >> np.uint64(16), tor.LOWEST_R, True)
    return out


@pytest.mark.parametrize("clip", [None, 0.37])
def test_adamw_8bit_codes_are_those_of_the_formulas_in_fp32(clip):
    """Every code and scale, over blocks whose magnitudes lie 24 decades apart (those that take 2^-120 first among them) with
    elements spread over five more."""
    table = wl.make_table([("a", (301, 1001)), ("v", (257,)), ("b", (64, 1024))])
    layers = H.layers_of(table)
    ctx = binding.Context(table, 1)
    d, x, m, v = _inputs(table, 41)
    g = torch.Generator(device="cuda").manual_seed(42)
    size = 10.0 ** (24.0 * torch.rand((table.stride + 255) // 256, generator=g, device="cuda") - 12.0)
    size = size.repeat_interleave(256)[:table.stride]
    d, m, v = d * size, m * size, v * size * size
    state, step, hyper = _pack(table, ctx, m, v), torch.tensor([20], device="cuda"), _hyper()
    factor = None if clip is None else torch.tensor([clip], device="cuda")
    f = 1.0 if clip is None else float(np.float32(clip))
    for k in range(3):
        want = _codes_by_fp32(_np(d), [_bytes(t).copy() for t in state], 20 + k, _np(hyper), layers, 6, f)
        ctx.acc_adamw_8bit(d, x, *state, step, hyper, seed=6, grad_scale=factor)
        assert all(np.array_equal(_bytes(t), w) for t, w in zip(state, want))
        d = d.roll(256)


@pytest.mark.parametrize("top", [1.0, 1e5, 1e18])
def test_adamw_8bit_a_positive_r_is_never_zero(top):
    """One element far above the others of its block: their r is under the grid (and, scaled, under fp32's range), and still
    gets the smallest code, also where the state before had one."""
    table = wl.make_table([("x", (3 * 256 + 17,))])
    ctx = binding.Context(table, 1)
    d = torch.full((table.stride,), 1e-10, device="cuda")
    d[::256] = top
    d[7] = 0.0
    state, x, step = ctx.new_adamw_8bit(), torch.zeros(table.stride, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    for _ in range(3):
        ctx.acc_adamw_8bit(d, x, *state, step, _hyper(), seed=1)
        r = _bytes(state[1])[:3 * 256 + 17]
        assert r[7] == 0 and (np.delete(r, 7) > 0).all()
