"""The pipeline's head and linear-layer classes with layouts whose workers and tokens are no single run of rows: nothing is copied
behind the caller's back, and nothing runs on another stream than the one given."""
import pytest
import torch

from paper_2010_16248_b200 import binding, pipeline, workloads as wl

pytestmark = pytest.mark.gpu


def _head(W, n, dtype, top=0):
    table = wl.make_table(wl.shapes_lstm(211, 26))
    ctx = binding.Context(table, W)
    return table, pipeline.TokenHead(ctx, "decoder.weight", n, dtype=dtype, top=top)


def _layouts(W, n, width, dtype, g):
    """``[W, n, width]`` views of other tensors: all but the last token, all but the first, tokens outermost."""
    wide = torch.randn(W, n + 1, width, generator=g, device="cuda").to(dtype)
    outer = torch.randn(n, W, width, generator=g, device="cuda").to(dtype)
    return wide[:, :-1], wide[:, 1:], outer.transpose(0, 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", [0, 1, 2])
@pytest.mark.parametrize("one", [False, True])
def test_layouts_without_copies(dtype, layout, one):
    W, n = 3, 17
    table, head = _head(W, n, dtype, top=4)
    _, want = _head(W, n, dtype, top=4)
    g = torch.Generator(device="cuda").manual_seed(layout)
    hidden, logits = (_layouts(W, n, width, dtype, g)[layout] for width in (head.cols, head.rows))
    tokens = torch.randint(-1, head.rows, (W, n), generator=g, device="cuda")
    g_logp = torch.full((1,), -0.25, device="cuda") if one else torch.randn(W, n, generator=g, device="cuda")
    g_entropy = torch.randn(W, n, generator=g, device="cuda")
    grads = [torch.zeros(W, table.stride, device="cuda") for _ in range(2)]
    # (a row's sums are taken in an order that goes by its start in memory: the same rows, worker by worker)
    for w in range(W):
        rows = slice(w * n, (w + 1) * n)
        ctx = want.ctx
        ctx.acc_checkpoint_store(hidden[w], want.code[rows], want.code_scale[rows], tokens[w])
        ctx.acc_token_logprobs(logits[w], tokens[w], want.logp[w], want.norm[w], want.entropy[w], want.top_index[rows],
                               want.top_logp[rows])
        ctx.acc_token_logprobs_grad(logits[w], tokens[w], want.norm[w], want.dlogits[w], g_logp if one else g_logp[w],
                                    g_entropy[w], want.entropy[w])
    want.backward(want.dlogits, grads[0])
    # what is queued on the current stream has nothing to do with the calls on the other one
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    torch.cuda._sleep(40_000_000)
    launches = [head.keep(hidden, tokens, side), head.forward(logits, tokens, side),
                head.backward_logits(logits, tokens, g_logp, g_entropy, side), head.backward(head.dlogits, grads[1], side)]
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    side.synchronize()
    for name in ("code", "code_scale", "logp", "entropy", "norm", "top_index", "top_logp", "dlogits"):
        a, b = (getattr(x, name).contiguous().view(torch.uint8) for x in (head, want))
        assert torch.equal(a, b), name
    assert torch.equal(*grads)
    assert launches[:3] == [W] * 3
    torch.cuda.synchronize()


def test_one_launch_where_the_rows_are_one_run():
    W, n = 3, 17
    _, head = _head(W, n, torch.bfloat16)
    tokens = torch.zeros(W, n, dtype=torch.int64, device="cuda")
    hidden = torch.zeros(W * n, head.cols, device="cuda")
    for x in (hidden, hidden.view(W, n, -1), torch.zeros(W, n, head.cols + 3, device="cuda")[:, :, :head.cols]):
        assert head.keep(x, tokens) == 1
    for z in (torch.zeros(W, n, head.rows, device="cuda"), head.new_logits(), torch.zeros(W * n, head.rows, device="cuda")):
        assert head.forward(z, tokens) == 1 and head.backward_logits(z, tokens, torch.ones(1, device="cuda")) == 1


def test_refusals():
    """Sizes that do not fit are refused for such layouts too."""
    W, n = 3, 17
    _, head = _head(W, n, torch.float32)
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    tokens = torch.zeros(W, n, dtype=torch.int64, device="cuda")
    for x, t in ((f(W, n + 2, head.cols)[:, :-1], tokens), (f(W + 1, n + 1, head.cols)[:, :-1], tokens),
                 (f(W, n + 1, head.cols)[:, :-1], tokens[:, 1:].contiguous()), (f(W, n + 1, head.cols)[:, :-1], f(W, n)),
                 (f(W, n + 1, head.cols)[:, :-1], torch.zeros(W, n + 1, dtype=torch.int64, device="cuda")[:, :-1]),
                 (f(W, n + 1, head.cols)[:, :-1], torch.zeros(W, n + 1, dtype=torch.int64, device="cuda")),
                 (f(W, head.cols, n).transpose(1, 2), tokens), (f(W, n + 1, head.cols + 1)[:, :-1], tokens)):
        with pytest.raises((ValueError, binding.AccError)):
            head.keep(x, t)
    z = f(W, n + 1, head.rows)[:, :-1]
    for a in ((f(W, n + 2, head.rows)[:, :-1], tokens), (z, tokens[:, 1:].contiguous()), (z, None)):
        with pytest.raises((ValueError, binding.AccError)):
            head.forward(*a)
    for g in (f(n), f(W, n + 1), f(W, n + 1)[:, :-1], f(W, n).double()):
        with pytest.raises((ValueError, binding.AccError)):
            head.backward_logits(z, tokens, g)
        with pytest.raises((ValueError, binding.AccError)):
            head.backward_logits(z, tokens, f(1), g)
