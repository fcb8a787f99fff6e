"""The head's operators as they are used together: hidden states kept in 8 bits, logits by a matrix product, log probabilities,
their gradient, the decoder's weight gradient, the compression step and AdamW; called one by one and through the pipeline's
classes, eager and as a replayed graph; and the loss's gradient with respect to the decoder against differences."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as hor
from paper_2010_16248_b200 import binding, pipeline, workloads as wl
from tests import helpers as H

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _slice(table, layer):
    o = int(table.offset[layer])
    return slice(o, o + int(table.rows[layer]) * int(table.cols[layer]))


@pytest.mark.parametrize("vocab,hidden,n,dtype", [(211, 26, 50, torch.float32), (1203, 40, 33, torch.bfloat16)])
def test_hidden_states_to_parameters(vocab, hidden, n, dtype):
    table, W = wl.make_table(wl.shapes_lstm(vocab, hidden)), 2
    ctx = binding.Context(table, W)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    params = torch.randn(table.stride, generator=g, device="cuda") * 0.1
    low = torch.zeros(table.stride, dtype=torch.bfloat16, device="cuda")
    opt = pipeline.AdamW(ctx, params, 1e-2, max_norm=1.0, params_bf16=low)
    head = pipeline.TokenHead(ctx, "decoder.weight", n, temperature=0.8, top=5, dtype=dtype)
    sl = _slice(table, head.layer)
    level = torch.ones(table.n_layers, dtype=torch.uint8, device="cuda")
    err, out = torch.zeros(W, table.stride, device="cuda"), torch.zeros(table.stride, device="cuda")
    q, p = ctx.new_q(wl.initial_q(table, 2, device="cuda")), ctx.new_p()
    tokens = torch.randint(0, vocab, (W, n), generator=g, device="cuda")
    tokens[:, ::7] = -1
    x = torch.randn(W, n, hidden, generator=g, device="cuda").to(dtype)
    x[:, ::7] = float("nan")  # padded positions
    g_logp, g_entropy = torch.full((1,), -1.0 / n, device="cuda"), torch.full((1,), -0.01, device="cuda")
    losses = []
    for it in range(3):
        head.keep(x, tokens)
        kept = head.kept(torch.empty_like(x))
        want = hor.checkpoint_decode(*hor.checkpoint_encode(x.view(-1, hidden).double().cpu().numpy(), tokens.view(-1).cpu().numpy()),
                                     hidden)
        assert np.array_equal(kept.view(-1, hidden).double().cpu().numpy(), want)
        logits = head.new_logits()
        logits.copy_(torch.matmul(kept.float(), params[sl].view(vocab, hidden).t()))
        head.forward(logits, tokens)
        z, t, scale = logits.reshape(-1, vocab).double().cpu().numpy(), tokens.view(-1).cpu().numpy(), float(np.float32(1.0 / 0.8))
        r = hor.token_logprobs(z, t, scale, 5)
        assert np.allclose(head.logp.view(-1).cpu().numpy(), r["logp"], rtol=1e-5, atol=1e-5)
        assert np.array_equal(head.top_index.cpu().numpy(), r["top_index"])
        losses.append(float(head.logp.sum()))
        head.backward_logits(logits, tokens, g_logp, g_entropy)
        dz = hor.token_logprobs_grad(z, t, head.norm.view(-1, 2).double().cpu().numpy(), np.full(W * n, float(g_logp)),
                                     np.full(W * n, float(g_entropy)), head.entropy.view(-1).double().cpu().numpy(), scale)
        half = 2.0 ** -8 if dtype == torch.bfloat16 else U
        assert (np.abs(head.dlogits.reshape(-1, vocab).double().cpu().numpy() - dz) <= half * np.abs(dz) * 1.01 + 3e-6 / n).all()
        grads = torch.zeros(W, table.stride, device="cuda")
        head.backward(head.dlogits, grads)
        for w in range(W):
            G, S = hor.linear_grad(head.dlogits[w].double().cpu().numpy(), kept[w].double().cpu().numpy(), 1.0)
            terms = n * (3 if dtype == torch.float32 else 1) + 40
            assert (np.abs(grads[w, sl].view(vocab, hidden).double().cpu().numpy() - G) <= 2 * U * (terms + 1) * S).all()
        assert not grads[:, :sl.start].any() and not grads[:, sl.stop:].any()
        e0, q0 = err.clone(), q.clone()
        ctx.acc_powersgd_step(grads, err, q, p, level, out)
        if it == 0:  # (the layers without a gradient are zeros; with rank 2 the decoder's is not)
            only = wl.make_table([(table.names[head.layer], (vocab, hidden))])
            assert only.n_layers == 1 and torch.isfinite(out[sl]).all() and out[sl].any()
            assert torch.allclose(err[:, sl], grads[:, sl] - out[sl], rtol=0, atol=1e-6)
        before = params[sl].clone()
        opt.step(out)
        assert torch.isfinite(params).all() and not torch.equal(before, params[sl])
        assert torch.equal(low[sl], params[sl].bfloat16())
    assert ctx.acc_device_status() == 0 and all(np.isfinite(losses))


def test_the_decoders_gradient_equals_differences_of_the_loss():
    """d loss / d W of the whole chain, at a few entries, against differences of the loss in fp64 on the kept input.

    The chain's gradient is off by rounding (fp32 throughout): 1e-5 of its largest entry; the differences by about 1e-9."""
    vocab, hidden, n, W = 97, 24, 40, 2
    table = wl.make_table([("w", (vocab, hidden))])
    ctx = binding.Context(table, W)
    g = torch.Generator(device="cuda").manual_seed(0)
    weight = torch.randn(vocab, hidden, generator=g, device="cuda") * 0.3
    head = pipeline.TokenHead(ctx, "w", n, dtype=torch.float32)
    tokens = torch.randint(0, vocab, (W, n), generator=g, device="cuda")
    head.keep(torch.randn(W, n, hidden, generator=g, device="cuda"))
    x = head.kept(torch.empty(W, n, hidden, device="cuda"))
    weights = torch.randn(W, n, generator=g, device="cuda")

    def loss(matrix, w):
        logp = torch.log_softmax(x[w].double() @ matrix.t(), 1)
        ent = torch.special.entr(logp.exp()).sum(1)
        return float((weights[w].double() * logp.gather(1, tokens[w][:, None])[:, 0]).sum() + 0.3 * ent.sum())

    logits = head.new_logits().copy_((x.double() @ weight.double().t()).float())
    head.forward(logits, tokens)
    head.backward_logits(logits, tokens, weights, torch.full((1,), 0.3, device="cuda"))
    grads = torch.zeros(W, table.stride, device="cuda")
    head.backward(head.dlogits, grads)
    got = grads[:, :vocab * hidden].view(W, vocab, hidden).double()
    for w in range(W):
        for r, c in ((0, 0), (5, 23), (96, 7), (int(tokens[w, 0]), 3), (50, 12)):
            a, b, eps = weight.double().clone(), weight.double().clone(), 1e-5
            a[r, c] += eps
            b[r, c] -= eps
            assert abs((loss(a, w) - loss(b, w)) / (2 * eps) - float(got[w, r, c])) <= 1e-5 * float(got.abs().max()) + 1e-8


@pytest.mark.parametrize("compressors", [("powersgd",), ("topk",), ("powersgd", "topk")])
def test_engine_with_a_head_equals_the_calls_and_its_graph(compressors):
    w = wl.workload(5, scale=40)
    table, W, n = w.table, w.n_workers, 30
    batch = wl.head_batch(w, n, device="cuda")
    kw = dict(rank_low=2, rank_high=1, check_every=3, q_init=wl.initial_q(table, 2, device="cuda"), overlap=False, head=batch)
    eager, graph = (pipeline.AccordionStep(table, W, compressors, **kw) for _ in range(2))
    ctx = binding.Context(table, W)
    head = pipeline.TokenHead(ctx, batch["layer"], n)
    sl = _slice(table, head.layer)
    stream = wl.GradientStream(w, device="cuda")
    bufs = [stream.grads(t).clone() for t in range(2)]
    plain = [b.clone() for b in bufs]
    for b in plain:
        head.keep(batch["hidden"], batch["tokens"])
        head.forward(batch["logits"], batch["tokens"])
        head.backward_logits(batch["logits"], batch["tokens"], batch["g_logp"])
        head.backward(head.dlogits, b)
    with_graph = [b.clone() for b in bufs]
    for t in range(4):
        eager.step(bufs[t % 2])
    graph.capture_graphs(with_graph)
    for buf in with_graph:
        buf[:, sl] = 0
    # (the capture's warm state is its own: only what a step makes of its inputs is compared)
    for t in range(4):
        graph.step_graph(t % 2)
    torch.cuda.synchronize()
    for k in range(2):
        assert torch.equal(bufs[k], plain[k]) and torch.equal(with_graph[k], plain[k])
    assert torch.equal(eager.head.logp, head.logp) and torch.equal(graph.head.logp, head.logp)
    for a, b in zip(eager.outputs(), graph.outputs()):
        assert torch.equal(a, b)
    assert eager.launches == graph.launches
    assert eager.ctx.acc_device_status() == 0 and graph.ctx.acc_device_status() == 0


def test_calls_behind_torch_kernels_and_copies():
    """Every call right behind kernels and copies that write its inputs, on one stream, without waits: the same bits as with."""
    table = wl.make_table([("w", (700, 96))])
    W, n = 2, 300
    ctx = binding.Context(table, W)
    head = pipeline.TokenHead(ctx, "w", n)
    g = torch.Generator(device="cuda").manual_seed(1)
    src = torch.randn(W, n, 96, generator=g, device="cuda")
    z = torch.randn(W, n, 700, generator=g, device="cuda") * 2
    tokens = torch.randint(0, 700, (W, n), generator=g, device="cuda")
    one = torch.full((1,), -1.0 / n, device="cuda")
    results = []
    for waits in (True, False):
        x, logits, grads = torch.zeros_like(src), head.new_logits(), torch.zeros(W, table.stride, device="cuda")
        for k in range(5):
            wait = torch.cuda.synchronize if waits else (lambda: None)
            x.copy_(src * (k + 1))
            wait()
            head.keep(x, tokens)
            wait()
            logits.copy_(z * (1 + 0.1 * k))
            wait()
            head.forward(logits, tokens)
            wait()
            head.backward_logits(logits, tokens, one)
            wait()
            grads.zero_()
            wait()
            head.backward(head.dlogits, grads)
            wait()
            grads.mul_(0.5)
            wait()
        torch.cuda.synchronize()
        results.append((grads.clone(), head.logp.clone(), head.dlogits.clone(), head.code.view(torch.uint8).clone()))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_many_rows_of_a_middling_vocabulary():
    """Where a warp takes a row although the row is longer than the shortest ones."""
    ctx = binding.Context(wl.make_table([("w", (8, 8))]), 1)
    n, vocab, top = 5000, 1501, 20
    g = torch.Generator(device="cuda").manual_seed(2)
    for kind in ("plain", "ties", "lowest"):
        z = torch.randn(n, vocab, generator=g, device="cuda")
        if kind == "ties":
            z = z.round()
        if kind == "lowest":
            z = torch.where(torch.rand(n, vocab, generator=g, device="cuda") < 0.005, z, torch.finfo(torch.float32).min)
        tokens = torch.randint(0, vocab, (n,), generator=g, device="cuda")
        f = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        index, logp, norm, ent, alt = torch.empty(n, top, dtype=torch.int32, device="cuda"), f(n), f(n, 2), f(n), f(n, top)
        ctx.acc_token_logprobs(z, tokens, logp, norm, ent, index, alt)
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(index.long(), order)
        want = torch.log_softmax(z.double(), 1)
        far = z.gather(1, tokens[:, None])[:, 0] > -1e30
        assert torch.allclose(logp[far].double(), want.gather(1, tokens[:, None])[:, 0][far], rtol=1e-5, atol=1e-5)
        entropy = torch.special.entr(want.exp()).sum(1)
        assert torch.allclose(ent.double(), entropy, rtol=1e-5, atol=1e-5)
        dz, g_logp, g_ent = f(n, vocab), torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
        ctx.acc_token_logprobs_grad(z, tokens, norm, dz, g_logp, g_ent, ent)
        p = want.exp()
        ref = -p * (g_logp.double()[:, None] + g_ent.double()[:, None] * (want.clamp(min=-1e300) * (p > 0) + entropy[:, None]))
        ref.scatter_add_(1, tokens[:, None], g_logp.double()[:, None])
        assert torch.allclose(dz.double(), ref, rtol=1e-4, atol=1e-6)


def test_refusals_of_the_classes():
    table = wl.make_table([("w", (20, 12)), ("v", (5,))])
    ctx = binding.Context(table, 2)
    with pytest.raises(ValueError):
        pipeline.TokenHead(ctx, "nothing", 4)
    with pytest.raises(binding.AccError):
        pipeline.CheckpointedLinear(ctx, "v", 4)
    head = pipeline.TokenHead(ctx, "w", 4)
    tokens = torch.zeros(2, 4, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        head.forward(head.new_logits(), tokens[:1])
    with pytest.raises(ValueError):
        head.keep(torch.zeros(2, 3, 12, device="cuda"))
    with pytest.raises(ValueError):
        head.backward(head.dlogits[:, :3], torch.zeros(2, table.stride, device="cuda"))
