"""A linear layer's weight gradient from an 8-bit checkpoint against the fp64 oracle on the decoded values, through the C-ABI.

Tolerance: products of bf16 terms are exact in fp32 (fp32 values of dy are three terms that add up to all 24 bits).  A sum of n
tokens (3 n terms for fp32) and its joins passes at most as many additions, each off by at most 2 u of the sum of the
magnitudes (u = 2^-24: a tensor core may cut instead of round); the scale and the addition to what is there are one rounding
each.
"""
import numpy as np
import pytest
import torch

from oracle import head_oracle as hor
from paper_2010_16248_b200 import binding, workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _ctx(rows, cols, W):
    """The layer in the middle of three, so that neighbours would show a stray write."""
    table = wl.make_table([("v", (5,)), ("layer", (rows, cols)), ("after", (3, 7))])
    return table, binding.Context(table, W), 1


def _slice(table, layer):
    o = int(table.offset[layer])
    return slice(o, o + int(table.rows[layer]) * int(table.cols[layer]))


def _inputs(W, n, rows, cols, ld, dtype, seed, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((offset + W * n * ld + rows,), float("nan"), dtype=dtype, device="cuda")
    dy = flat[offset:offset + W * n * ld].view(W, n, ld)[:, :, :rows]
    size = 10.0 ** (-3.0 * torch.rand(W, n, 1, generator=g, device="cuda"))
    dy.copy_(torch.randn(W, n, rows, generator=g, device="cuda") * size)
    x = torch.randn(W * n, cols, generator=g, device="cuda") * 10.0 ** (2 * torch.rand(cols, generator=g, device="cuda") - 1)
    return dy, x


def _check(table, ctx, layer, dy, x, scale=1.0, accumulate=False):
    W, n, rows = dy.shape
    cols = x.shape[1]
    code, scales = ctx.new_checkpoint(W * n, cols)
    ctx.acc_checkpoint_store(x, code, scales)
    values = hor.checkpoint_decode(code.view(torch.uint8).cpu().numpy(), scales.view(torch.uint8).cpu().numpy(), cols)
    grads = torch.randn(W, table.stride, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda")
    before = grads.clone()
    ws = ctx.new_linear_grad_workspace(layer, n)
    ws.fill_(0xFF)  # whatever was there
    ctx.acc_linear_grad(layer, dy, code, scales, grads, scale=scale, accumulate=accumulate, workspace=ws)
    assert ctx.acc_device_status() == 0
    sl = _slice(table, layer)
    terms = n * (3 if dy.dtype == torch.float32 else 1) + 40
    for w in range(W):
        got = grads[w, sl].view(rows, cols).double()
        d, v = dy[w].double(), torch.from_numpy(values[w * n:(w + 1) * n]).cuda()
        want, size = scale * (d.t() @ v), abs(scale) * (d.abs().t() @ v.abs())
        if rows * cols * n < 2_000_000:
            one, mag = hor.linear_grad(dy[w].double().cpu().numpy(), values[w * n:(w + 1) * n], scale)
            assert np.allclose(want.cpu().numpy(), one, rtol=1e-12, atol=1e-12 * (mag.max() if mag.size else 0))
        bound = (2 * U * terms + 2 * U) * size
        if accumulate:
            want = want + before[w, sl].view(rows, cols).double()
            bound = bound + U * (want.abs() + size)
        off = (got - want).abs()
        assert bool((off <= bound + 1e-37).all()), (w, float((off - bound).max()), int((off > bound).sum()))
        outside = torch.cat([grads[w, :sl.start] - before[w, :sl.start], grads[w, sl.stop:] - before[w, sl.stop:]])
        assert not outside.any()
    again = before.clone()
    ctx.acc_linear_grad(layer, dy, code, scales, again, scale=scale, accumulate=accumulate, workspace=ws)
    assert torch.equal(again, grads)
    return code, scales, grads


# (W, n, rows, cols): tiles and steps that end anywhere, several tiles a block, sums split over the tokens
SIZES = [(1, 1, 1, 1), (1, 64, 128, 256), (1, 16, 8, 16), (2, 3, 5, 7), (1, 65, 129, 257), (3, 100, 130, 33), (2, 35, 300, 650),
         (1, 128, 257, 1030), (1, 4000, 64, 16), (2, 1000, 33, 520), (1, 35, 2600, 650), (8, 200, 700, 130), (1, 2049, 600, 300),
         (3, 777, 1111, 97),
         # few tokens of layers too large for the kernel of few tokens; just within it; 65 tokens of a small one
         (8, 40, 2000, 650), (3, 1, 8000, 5000), (1, 64, 1250, 1250), (1, 65, 70, 90), (2, 64, 513, 67)]


@pytest.mark.parametrize("W,n,rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ld", ["wide", "contiguous", "odd"])
def test_linear_grad(W, n, rows, cols, dtype, ld):
    table, ctx, layer = _ctx(rows, cols, W)
    step = {"wide": (rows + 7) // 8 * 8, "contiguous": rows, "odd": rows + 1 - rows % 2 + 2}[ld]
    dy, x = _inputs(W, n, rows, cols, step, dtype, n + rows, offset=0 if ld != "odd" else 1)
    _check(table, ctx, layer, dy, x, scale=[1.0, 0.25, -3.0][n % 3], accumulate=(W + n) % 2 == 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_workers_inside_tokens_and_other_layouts(dtype):
    """dy as [n][W][rows], viewed as [W][n][rows]; a slice of wider rows; one worker of many."""
    table, ctx, layer = _ctx(200, 90, 3)
    g = torch.Generator(device="cuda").manual_seed(5)
    dy = torch.randn(50, 3, 208, generator=g, device="cuda").to(dtype)
    x = torch.randn(150, 90, generator=g, device="cuda")
    _check(table, ctx, layer, dy.transpose(0, 1)[:, :, :200], x)
    _check(table, ctx, layer, dy.transpose(0, 1)[:, :, 8:], x)
    _check(table, ctx, layer, dy.transpose(0, 1)[:, :, 3:203], x)


def test_zero_tokens():
    table, ctx, layer = _ctx(20, 30, 2)
    grads = torch.ones(2, table.stride, device="cuda")
    ws = ctx.new_linear_grad_workspace(layer, 0)
    code, scales = ctx.new_checkpoint(0, 30)
    dy = torch.zeros(2, 0, 20, device="cuda")
    ctx.acc_linear_grad(layer, dy, code, scales, grads, accumulate=True, workspace=ws)
    assert (grads == 1).all()
    ctx.acc_linear_grad(layer, dy, code, scales, grads, workspace=ws)
    sl = _slice(table, layer)
    assert not grads[:, sl].any() and (grads[:, :sl.start] == 1).all() and (grads[:, sl.stop:] == 1).all()


def test_infinities_and_nan_stay_in_their_rows_and_columns():
    for dtype in (torch.bfloat16, torch.float32):
        table, ctx, layer = _ctx(140, 70, 1)
        dy, x = _inputs(1, 90, 140, 70, 144, dtype, 3)
        x = x.abs() + 1
        dy[0, 5, 3], dy[0, 6, 100], dy[0, 7, 130] = float("inf"), float("nan"), -float("inf")
        x[9, 40] = float("nan")  # its block of 32 columns reads as NaN
        code, scales = ctx.new_checkpoint(90, 70)
        ctx.acc_checkpoint_store(x, code, scales)
        grads = torch.zeros(1, table.stride, device="cuda")
        ctx.acc_linear_grad(layer, dy, code, scales, grads, workspace=ctx.new_linear_grad_workspace(layer, 90))
        got = grads[0, _slice(table, layer)].view(140, 70)
        assert torch.isnan(got[:, 32:64]).all()
        rest = torch.cat([got[:, :32], got[:, 64:]], 1)
        assert (rest[3] == float("inf")).all() and torch.isnan(rest[100]).all() and (rest[130] == -float("inf")).all()
        rest[[3, 100, 130]] = 0
        assert torch.isfinite(rest).all()


def test_large_and_small_scales_of_the_checkpoint_are_exact():
    table, ctx, layer = _ctx(16, 64, 1)
    x = torch.zeros(3, 64, device="cuda")
    x[0, :32], x[0, 32:] = 1.5e30, 2.0 ** -110
    x[1, 5], x[2, 40] = 448.0, 3.0e-30
    dy = torch.zeros(1, 3, 16, dtype=torch.bfloat16, device="cuda")
    dy[0, 0, 0] = dy[0, 1, 1] = dy[0, 2, 2] = 1.0
    code, scales = ctx.new_checkpoint(3, 64)
    ctx.acc_checkpoint_store(x, code, scales)
    values = torch.empty(3, 64, device="cuda")
    ctx.acc_checkpoint_load(code, scales, values)
    grads = torch.zeros(1, table.stride, device="cuda")
    ctx.acc_linear_grad(layer, dy, code, scales, grads, workspace=ctx.new_linear_grad_workspace(layer, 3))
    assert torch.equal(grads[0, _slice(table, layer)].view(16, 64)[:3], values)


def test_streams_and_graphs():
    table, ctx, layer = _ctx(500, 300, 2)
    dy, x = _inputs(2, 500, 500, 300, 504, torch.bfloat16, 1)
    code, scales, want = _check(table, ctx, layer, dy, x)
    got = [torch.zeros_like(want) for _ in range(2)]
    ws = [ctx.new_linear_grad_workspace(layer, 500) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for g, w, s in zip(got, ws, streams):
            ctx.acc_linear_grad(layer, dy, code, scales, g, workspace=w, stream=s)
    torch.cuda.synchronize()
    sl = _slice(table, layer)
    assert all(torch.equal(g[:, sl], want[:, sl]) for g in got)
    static, out = dy.clone(), torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.acc_linear_grad(layer, static, code, scales, out, workspace=ws[0])
    for factor in (2.0, 1.0):
        static.copy_(dy * factor)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:, sl], want[:, sl] * factor)


def test_refusals():
    table, ctx, layer = _ctx(20, 30, 2)
    lib = binding.lib()
    dy = torch.zeros(2, 6, 20, device="cuda")
    code, scales = ctx.new_checkpoint(12, 30)
    grads, ws = torch.zeros(2, table.stride, device="cuda"), ctx.new_linear_grad_workspace(layer, 6)
    for a in ((0, dy), (3, dy), (-1, dy), (layer, dy.half()), (layer, dy[0]), (layer, dy[:1]), (layer, dy[:, :, :19]), (layer, dy.cpu()),
              (layer, dy[:, :5])):
        with pytest.raises(ValueError):
            ctx.acc_linear_grad(*a, code, scales, grads, workspace=ws)
    for a in ((code[:11], scales, grads), (code, scales[:11], grads), (code, scales, grads[:1]), (code, scales, grads.double()),
              (code.view(torch.uint8), scales, grads), (code, scales.cpu(), grads)):
        with pytest.raises(ValueError):
            ctx.acc_linear_grad(layer, dy, *a, workspace=ws)
    for w, status in ((None, 3), (ws[:-1], 3), (torch.zeros(ws.numel() + 256, dtype=torch.uint8, device="cuda")[16:], 2)):
        with pytest.raises(binding.AccError) as e:
            ctx.acc_linear_grad(layer, dy, code, scales, grads, workspace=w)
        assert e.value.status == status
    with pytest.raises(binding.AccError) as e:  # workers that share their rows
        ctx.acc_linear_grad(layer, dy[:1].expand(2, 6, 20), code, scales, grads, workspace=ws)
    assert e.value.status == 1
    d, c, s, g, w, n = dy.data_ptr(), code.data_ptr(), scales.data_ptr(), grads.data_ptr(), ws.data_ptr(), ws.numel()
    call = lambda **k: lib.acc_linear_grad(ctx._h, *{**dict(layer=layer, dy=d, dt=0, n=6, ld=20, st=120, f=1.0, c=c, s=s, g=g, acc=0,  # noqa: E731
                                                            w=w, nb=n), **k}.values(), None)
    assert [call(dt=2), call(n=-1), call(n=(1 << 27) + 1, nb=1 << 40), call(ld=19), call(st=19), call(dy=None), call(c=None), call(s=None),
            call(g=None)] == [1] * 9
    assert [call(dy=d + 2), call(c=c + 8), call(g=g + 4)] == [2] * 3
