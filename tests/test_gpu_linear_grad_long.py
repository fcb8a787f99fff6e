"""A linear layer's weight gradient over very many tokens, through the C-ABI."""
import pytest
import torch

from paper_2010_16248_b200 import binding, workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,ld", [(torch.bfloat16, 8), (torch.bfloat16, 1), (torch.float32, 1)])
def test_as_many_tokens_as_there_may_be(dtype, ld):
    """2^28 tokens (131072 steps in each of 32 splits, whose parts are found by products beyond 32 bits) of a layer of one element.
    Ones times codes of 1: every partial sum is a whole number below 2^24 or a sum of a few multiples of 2^23, so exact."""
    n = 1 << 28
    ctx = binding.Context(wl.make_table([("layer", (1, 1))]), 1)
    dy = torch.zeros(1, n, ld, dtype=dtype, device="cuda")[:, :, :1]
    dy.fill_(1.0)
    code, scale = ctx.new_checkpoint(n, 1)
    code.view(torch.uint8)[:, 0] = 0x38  # 1
    scale.view(torch.uint8).fill_(127)   # 2^0
    grads = torch.zeros(1, int(ctx.stride), device="cuda")
    workspace = ctx.new_linear_grad_workspace(0, n)
    ctx.acc_linear_grad(0, dy, code, scale, grads, workspace=workspace)
    assert ctx.acc_device_status() == 0
    assert float(grads[0, 0]) == float(n)
    # the last token alone
    dy.zero_()
    dy[0, -1] = 3.0
    ctx.acc_linear_grad(0, dy, code, scale, grads, workspace=workspace)
    assert ctx.acc_device_status() == 0 and float(grads[0, 0]) == 3.0


@pytest.mark.parametrize("dtype,extra", [(torch.bfloat16, 0), (torch.bfloat16, 1), (torch.float32, 0), (torch.float32, 1)])
def test_no_long_sum_stays_in_the_tensor_core(dtype, extra):
    """16384 tokens of one sign into a layer of as many tiles as there are pairs of SMs, so that no split shortens the sums.  The
    tensor core cuts each of its additions by up to a unit in the last place, 2^-23 of the sum so far.  Of 24 products that add up
    evenly that is (24 + 1) / 2 of 2^-23; of an fp32 dy's, whose terms of little size come after four of much, 1.25 + 4 + 3.25 + 8 =
    16.5; half a unit more for what is uneven.  The sums (of 6 steps of 64 tokens, of 2) are added up in fp32, each off by half a
    unit.  (A single sum of all products, tried, is 1.5e-5 off, 1.2e-4 in fp32.)"""
    n, rows, cols = 16384, 256 * 74, 32
    ctx = binding.Context(wl.make_table([("layer", (rows, cols))]), 1)
    workspace = ctx.new_linear_grad_workspace(0, n)
    assert workspace.numel() == 2 * cols * n  # the decoded checkpoint alone: one split
    g = torch.Generator(device="cuda").manual_seed(extra)
    dy = torch.empty(1, n, rows + extra, dtype=dtype, device="cuda")[:, :, :rows]
    for k in range(0, n, 2048):
        dy[0, k:k + 2048] = (torch.rand(2048, rows, generator=g, device="cuda") + 0.5).to(dtype)
    x = torch.rand(n, cols, generator=g, device="cuda") + 0.5
    code, scale = ctx.new_checkpoint(n, cols)
    ctx.acc_checkpoint_store(x, code, scale)
    ctx.acc_checkpoint_load(code, scale, x)
    grads = torch.zeros(1, int(ctx.stride), device="cuda")
    ctx.acc_linear_grad(0, dy, code, scale, grads, workspace=workspace)
    assert ctx.acc_device_status() == 0
    want = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    for k in range(0, n, 2048):
        want += dy[0, k:k + 2048].double().t() @ x[k:k + 2048].double()
    sums = 43 if dtype is torch.bfloat16 else 128
    bound = (13.0 if dtype is torch.bfloat16 else 17.0) * 2.0 ** -23 + (sums + 1) / 2 * 2.0 ** -24 + 2.0 ** -24
    off = float(((grads[0, :rows * cols].view(rows, cols).double() - want).abs() / want).max())
    assert off <= bound, (off, bound)
