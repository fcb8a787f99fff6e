"""8-bit activation checkpoints against the fp64 oracle: codes and scales bit for bit, values exactly (fp32) or rounded once."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as hor
from paper_2010_16248_b200 import binding, workloads as wl

pytestmark = pytest.mark.gpu


def _ctx():
    return binding.Context(wl.make_table([("layer", (8, 40))]), 1)


def _rows(n, cols, ld, dtype, offset=0, fill=float("nan")):
    flat = torch.full((offset + n * ld + cols,), fill, dtype=dtype, device="cuda")
    return flat, flat[offset:offset + n * ld].view(n, ld)[:, :cols]


def _values(rng, n, cols, dtype):
    """Magnitudes from the type's least to its largest, zeros, blocks of zeros, a block of NaN and one of infinities."""
    x = rng.normal(0, 1, (n, cols)) * 10.0 ** rng.uniform(-2, 2, (n, cols)) * 10.0 ** rng.uniform(-12, 12, (n, 1))
    x[rng.random((n, cols)) < 0.05] = 0
    t = torch.from_numpy(x).to(dtype)
    if n > 5:
        t[0] = 0
        t[1, ::3] = torch.finfo(dtype).smallest_normal / 4
        t[2, cols // 2] = torch.finfo(dtype).max
        t[3, cols - 1] = float("nan")
        t[4, 0] = -float("inf")
        t[5] = -0.0
    return t


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


SIZES = [(1, 1, 1), (2, 3, 5), (9, 31, 31), (7, 32, 32), (6, 33, 34), (700, 650, 650), (33, 650, 656), (50, 650, 651), (5, 1000, 1000),
         (1, 8192, 8192), (3, 8191, 8200), (10000, 8, 8), (2000, 40, 48)]


@pytest.mark.parametrize("n,cols,ld", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("padded", [False, True])
def test_store_and_load(n, cols, ld, dtype, padded):
    rng = np.random.default_rng(n + cols)
    ctx = _ctx()
    _, x = _rows(n, cols, ld, dtype, offset=cols % 3)
    x.copy_(_values(rng, n, cols, dtype))
    tokens = np.where(rng.random(n) < 0.4, -2, 5) if padded else None
    dev = None if tokens is None else torch.from_numpy(tokens).to([torch.int32, torch.int64][n % 2]).cuda()
    if padded:
        x[dev < 0] = float("nan")
    code, scale = ctx.new_checkpoint(n, cols)
    code.view(torch.uint8).fill_(0x55), scale.view(torch.uint8).fill_(0x55)
    ctx.acc_checkpoint_store(x, code, scale, tokens=dev)
    want_code, want_byte = hor.checkpoint_encode(x.double().cpu().numpy(), tokens)
    assert np.array_equal(_bytes(scale), want_byte)
    assert np.array_equal(_bytes(code), want_code)
    values = hor.checkpoint_decode(want_code, want_byte, cols)
    for out_type in (torch.float32, torch.bfloat16):
        flat, out = _rows(n, cols, ld, out_type, offset=cols % 3, fill=9.0)
        ctx.acc_checkpoint_load(code, scale, out)
        want = torch.from_numpy(values).float().to(out_type).cuda()
        assert torch.equal(torch.nan_to_num(out, nan=3.0), torch.nan_to_num(want, nan=3.0))
        assert torch.equal(torch.isnan(out), torch.isnan(want))
        flat[cols % 3:cols % 3 + n * ld].view(n, ld)[:, :cols] = 9.0
        assert (flat == 9.0).all()
    assert ctx.acc_device_status() == 0


def test_every_code_and_scale_reads_back():
    ctx = _ctx()
    code, scale = ctx.new_checkpoint(8 * 255, 32)
    code.view(torch.uint8).copy_(torch.arange(256, dtype=torch.uint8, device="cuda").view(8, 32).repeat(255, 1))
    scale.view(torch.uint8).copy_(torch.arange(255, dtype=torch.uint8, device="cuda").repeat_interleave(8)[:, None])
    out = torch.empty(8 * 255, 32, device="cuda")
    ctx.acc_checkpoint_load(code, scale, out)
    want = code.double() * torch.from_numpy(2.0 ** (np.arange(255) - 127.0)).cuda().repeat_interleave(8)[:, None]
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(out), nan) and torch.equal(out[~nan], want.float()[~nan])


def test_ties_go_to_even():
    ctx = _ctx()
    x = torch.zeros(1, 32, device="cuda")
    x[0, 0] = 128.0
    half = torch.tensor([17, 19, 21, 23, 25, 27, 29, 31], device="cuda") / 16.0  # half-way between codes of [1, 2)
    x[0, 1:9], x[0, 9:17] = half, -half * 8
    x[0, 17:20] = torch.tensor([0.5, 1.5, 2.5], device="cuda") * 2.0 ** -9  # half-way between subnormal codes
    code, scale = ctx.new_checkpoint(1, 32)
    ctx.acc_checkpoint_store(x, code, scale)
    out = torch.empty_like(x)
    ctx.acc_checkpoint_load(code, scale, out)
    even = torch.tensor([16, 20, 20, 24, 24, 28, 28, 32], device="cuda") / 16.0
    assert torch.equal(out[0, 1:9], even) and torch.equal(out[0, 9:17], -even * 8)
    assert torch.equal(out[0, 17:20], torch.tensor([0.0, 2.0, 2.0], device="cuda") * 2.0 ** -9)


def test_rows_beyond_31_bits_and_graphs():
    ctx, n, cols = _ctx(), 524300, 4096  # 2.1e9 elements
    x = torch.zeros(n, cols, dtype=torch.bfloat16, device="cuda")
    x[-1] = 3.0
    code, scale = ctx.new_checkpoint(n, cols)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.acc_checkpoint_store(x, code, scale)
        ctx.acc_checkpoint_load(code, scale, x)
    for v in (3.0, 5.0):
        x[-1], x[-2] = v, 0
        code.view(torch.uint8)[-3:] = 1
        graph.replay()
        torch.cuda.synchronize()
        assert (x[-1] == v).all() and not x[-2].any() and (code[-1].float() == (64.0 if v < 4 else 32.0) * v).all()


def test_refusals():
    ctx, lib = _ctx(), binding.lib()
    x = torch.zeros(6, 40, device="cuda")
    code, scale = ctx.new_checkpoint(6, 40)
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    for a in ((x.half(), code, scale), (x[0], code, scale), (x.t(), code, scale), (x.cpu(), code, scale), (x, code[:5], scale),
              (x, code, scale[:, :1]), (x, code.view(torch.uint8), scale), (x, code, scale.view(torch.uint8)), (x, code.cpu(), scale),
              (x, None, scale)):
        with pytest.raises((ValueError, binding.AccError)):
            ctx.acc_checkpoint_store(*a)
        with pytest.raises((ValueError, binding.AccError)):
            ctx.acc_checkpoint_load(a[1], a[2], a[0])
    for tokens in (t[:5], t.float(), t.cpu(), [0] * 6):
        with pytest.raises(ValueError):
            ctx.acc_checkpoint_store(x, code, scale, tokens=tokens)
    with pytest.raises(binding.AccError) as e:
        ctx.acc_checkpoint_load(code, scale, x[:1].expand(6, 40))
    assert e.value.status == 1
    a, c, s = x.data_ptr(), code.data_ptr(), scale.data_ptr()
    assert lib.acc_checkpoint_store(ctx._h, a, 2, 6, 40, 40, None, 0, c, s, None) == 1
    assert lib.acc_checkpoint_store(ctx._h, a, 0, -1, 40, 40, None, 0, c, s, None) == 1
    assert lib.acc_checkpoint_store(ctx._h, a, 0, 6, 0, 40, None, 0, c, s, None) == 1
    assert lib.acc_checkpoint_store(ctx._h, a, 0, 6, 40, 39, None, 0, c, s, None) == 1
    assert lib.acc_checkpoint_store(ctx._h, a, 0, 6, 40, 40, t.data_ptr(), 3, c, s, None) == 1
    assert lib.acc_checkpoint_store(ctx._h, a, 0, (1 << 28) + 1, 40, 40, None, 0, c, s, None) == 1
    assert lib.acc_checkpoint_store(ctx._h, a + 2, 0, 5, 40, 40, None, 0, c, s, None) == 2
    assert lib.acc_checkpoint_store(ctx._h, a, 0, 5, 40, 40, None, 0, c + 8, s, None) == 2
    assert lib.acc_checkpoint_load(ctx._h, c, s, 5, 40, a + 1, 1, 40, None) == 2
    ctx.acc_checkpoint_store(x[:0], code[:0], scale[:0])
    assert ctx.last_launch_count() == 0
