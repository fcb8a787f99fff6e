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
