"""Log probabilities and their gradient of the longest rows that the calls take, whose last indices pass 2^31 by a step."""
import pytest
import torch

from paper_2010_16248_b200 import binding, workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [2 ** 31 - 17, 2 ** 31 - 2500])
@pytest.mark.parametrize("offset", [0, 1])  # rows of the result that start where the logits' do, and elsewhere (single elements)
def test_longest_rows(vocab, offset):
    ctx = binding.Context(wl.make_table([("decoder", (40, 8))]), 1)
    z = torch.zeros(1, vocab, dtype=torch.bfloat16, device="cuda")
    token = torch.tensor([vocab - 1], device="cuda")
    norm, logp, entropy = torch.empty(1, 2, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    ctx.acc_token_logprobs(z, token, logp=logp, norm=norm, entropy=entropy)
    # equal logits: the log of their number, whose sum in fp32 is exact but for its last rounding
    want = torch.tensor(float(vocab), dtype=torch.float64).log()
    for got in (norm[0, 1], -logp[0], entropy[0]):
        assert abs(float(got) - float(want)) < 1e-5
    flat = torch.full((vocab + 16,), 9.0, dtype=torch.bfloat16, device="cuda")
    out = flat[offset:offset + vocab].view(1, vocab)
    ctx.acc_token_logprobs_grad(z, token, norm, out, g_logp=torch.full((1,), 2.0 ** 31, device="cuda"))
    # -2^31 / vocab and 2^31 (1 - 1 / vocab), to bf16 both whole powers
    assert float(out[0, -1]) == 2.0 ** 31
    for part in out[0, :-1].split(1 << 28):
        assert bool((part == -1.0).all())
    assert bool((flat[:offset] == 9.0).all()) and bool((flat[offset + vocab:] == 9.0).all())
    assert ctx.acc_device_status() == 0
