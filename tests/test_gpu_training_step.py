"""The training operators as they are used together: lookup -> embedding gradient -> compression step -> norms, clip factor
and AdamW, called one by one and through the pipeline's classes, eager and as a replayed graph."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import accordion_oracle as orc
from oracle import training_oracle as tor
from paper_2010_16248_b200 import binding, pipeline, workloads as wl
from tests import helpers as H

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _lm(vocab=211, hidden=26):
    return wl.make_table(wl.shapes_lstm(vocab, hidden))


def _grads(table, W, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    mask = torch.zeros(table.stride, device="cuda")
    for _, sl in table.slices():
        mask[sl] = 1.0
    return torch.randn(W, table.stride, generator=g, device="cuda") * mask * 0.1


def _tokens(W, n, rows, seed, pad=True):
    rng = np.random.default_rng(seed)
    t = np.minimum((rng.pareto(0.8, (W, n)) * 2).astype(np.int64), rows - 1)
    if pad:
        t[rng.random((W, n)) < 0.1] = -1
    return torch.from_numpy(t).cuda()


@pytest.mark.parametrize("compressor", ["powersgd", "topk"])
@pytest.mark.parametrize("bits", [32, 8])
def test_token_to_parameter_run_matches_the_oracles(compressor, bits):
    """Two steps of a small language model's update, each stage checked against its oracle from the stage's own inputs."""
    table, W, n, scale = _lm(), 3, 50, 5.0
    layers = H.layers_of(table)
    rows, cols = 211, 26
    sl = slice(0, rows * cols)
    ctx = binding.Context(table, W, rank_low=2, rank_high=1, topk_low_bp=1000, topk_high_bp=100)
    g = torch.Generator(device="cuda").manual_seed(3)
    params = torch.randn(table.stride, generator=g, device="cuda") * 0.1
    level = torch.tensor([l % 2 for l in range(table.n_layers)], dtype=torch.uint8, device="cuda")
    err = torch.zeros(W, table.stride, device="cuda")
    q, p = ctx.new_q(wl.initial_q(table, 2, device="cuda")), ctx.new_p()
    vals, idx, counts = ctx.new_topk_buffers()
    out = torch.zeros(table.stride, device="cuda")
    opt = pipeline.AdamW(ctx, params, 1e-2, bits=bits, max_norm=0.5, decay_vectors=False, seed=7)
    emb = pipeline.TokenEmbedding(ctx, "encoder.weight", n, scale)
    hyper = opt.hyper.cpu().numpy()
    for it in range(2):
        tokens = _tokens(W, n, rows, it)
        y = torch.empty(W, n, cols, device="cuda")
        emb.lookup(params, tokens, y)
        want = tor.embedding_lookup(params[sl].view(rows, cols).cpu().numpy(), tokens.cpu().numpy(), scale)
        assert np.abs(y.view(-1, cols).cpu().numpy() - want).max() <= U * np.abs(want).max()
        dy = y * 0.01 + 0.02  # the gradient of a quadratic and a linear term
        grads = _grads(table, W, it)
        before = grads.clone()
        emb.backward(tokens, dy, grads)
        for w in range(W):
            G, S, K = tor.embedding_grad(tokens[w].cpu().numpy(), dy[w].cpu().numpy(), rows, scale)
            got = grads[w, sl].view(rows, cols).cpu().numpy()
            assert (np.abs(got - G) <= 1.01 * U * (np.maximum(K - 1, 0)[:, None] * S + 2 * np.abs(G))).all()
        assert torch.equal(grads[:, sl.stop:], before[:, sl.stop:])
        e0, q0 = err.clone(), q.clone()
        if compressor == "powersgd":
            ctx.acc_powersgd_step(grads, err, q, p, level, out)
            H.check_powersgd_against_oracle(ctx, table, grads, e0, q0, level, out, err, q, p, 2, 1, 1e-8)
        else:
            ctx.acc_topk_step(grads, err, level, vals, idx, counts, out)
            H.check_topk_against_oracle(ctx, table, grads, e0, level, vals, idx, counts, out, err, 1000, 100)
        x0 = params.cpu().numpy().copy()
        if bits == 32:
            m0, v0 = opt.m.cpu().numpy().copy(), opt.v.cpu().numpy().copy()
        else:
            m0, r0 = (tor.decode(c.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy(), layers)
                      for c, s in ((opt.m_code, opt.m_scale), (opt.r_code, opt.r_scale)))
            v0 = r0 * r0
        assert opt.step(out) == 4  # two for the norms, the factor, the update of a table this small
        factor, norm = tor.clip_factor(orc.layer_norms2(out.cpu().numpy(), layers), 0.5)
        assert abs(float(opt.factor) - factor) <= 2 * U * factor and abs(float(opt.norm) - norm) <= 1e-9 * norm
        X, M, V, T = tor.adamw(out.cpu().numpy(), x0, m0, v0, it, hyper, layers, float(opt.factor), decay_vectors=False)
        # (the update's error is at most 14 u of its size lr / (1 - beta1^t) * |m| / denominator <= lr / (1 - beta1^t) *
        # (1 / sqrt(1 - beta2)) at these two steps, and 2 u of the parameter: the element-wise bounds have their own tests)
        bound = 2 * U * np.abs(X) + 40 * U * 1e-2 / (1 - 0.9 ** T) * 32
        got = params.cpu().numpy()
        for (off, r, c, kind) in layers:
            s = slice(off, off + r * c)
            assert (np.abs(got[s] - X[s]) <= bound[s]).all()
        assert int(opt.step_count) == T
    assert ctx.acc_device_status() == 0


@pytest.mark.parametrize("compressor,bits,max_norm", [("powersgd", 32, 0.3), ("topk", 8, None)])
def test_accordion_step_with_adamw_and_embedding(compressor, bits, max_norm):
    """The engine gives the bits of the calls one by one, and its captured graphs those of the engine."""
    table, W, n = _lm(), 2, 40
    tokens, g = _tokens(W, n, 211, 9), torch.Generator(device="cuda").manual_seed(4)
    dy = torch.randn(W, n, 26, generator=g, device="cuda")
    x0 = torch.randn(table.stride, generator=g, device="cuda")
    ring = [_grads(table, W, 50 + k) for k in range(2)]

    def engine(accumulate=False):
        x, low = x0.clone(), torch.zeros(table.stride, dtype=torch.bfloat16, device="cuda")
        opt = {"kind": "adamw", "params": x, "lr": 0.01, "bits": bits, "max_norm": max_norm, "params_bf16": low, "seed": 5}
        emb = {"layer": "encoder.weight", "tokens": tokens, "dy": dy, "scale": 2.0, "accumulate": accumulate}
        return x, low, pipeline.AccordionStep(table, W, (compressor,), check_every=2, lazy_residual=True, optimizer=opt,
                                              embedding=emb)

    x, low, eng = engine()
    for k in range(4):
        eng.step(ring[k % 2].clone())
    ctx = binding.Context(table, W, flags=binding.ACC_FLAG_LAZY_RESIDUAL)
    y = x0.clone()
    opt = pipeline.AdamW(ctx, y, 0.01, bits=bits, max_norm=max_norm, seed=5)
    emb = pipeline.TokenEmbedding(ctx, "encoder.weight", n, 2.0)
    ref = pipeline.AccordionStep(table, W, (compressor,), check_every=2, lazy_residual=True)
    for k in range(4):
        grads = ring[k % 2].clone()
        emb.backward(tokens, dy, grads)
        ref.step(grads)
        opt.step(ref.outputs()[0])
    assert torch.equal(x, y) and not torch.equal(x, x0)
    cover = torch.zeros(table.stride, dtype=torch.bool, device="cuda")
    for _, sl in table.slices():
        cover[sl] = True
    assert torch.equal(low[cover], x[cover].to(torch.bfloat16))
    z, _, cap = engine()
    bufs = [r.clone() for r in ring]
    cap.capture_graphs(bufs)
    for k in range(4):
        bufs[k % 2].copy_(ring[k % 2])
        cap.step_graph(k % 2)
    torch.cuda.synchronize()
    assert torch.equal(x, z) and int(cap.adamw.step_count) == 4
    cap.set_lr(0.0)
    cap.adamw.hyper[4:].fill_(0.0)
    before = z.clone()
    cap.step_graph(0)
    torch.cuda.synchronize()
    assert torch.equal(before, z)  # the replayed graph reads the new rate
    _, _, acc = engine(accumulate=True)
    grads = ring[0].clone()
    acc.step(grads)
    want = ring[0].clone()
    ctx.acc_embedding_grad(0, tokens, dy, want, scale=2.0, accumulate=True, workspace=ctx.new_embedding_workspace(0, n))
    assert torch.equal(grads, want)


def test_batch_mode_and_real_workers_take_adamw():
    table, W = _lm(64, 12), 2
    x0 = torch.randn(table.stride, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    grads = [_grads(table, W, k) for k in range(2)]
    x, y = x0.clone(), x0.clone()
    batch = pipeline.BatchSizeStep(table, W, 2, 4, 1, optimizer={"kind": "adamw", "params": x, "lr": 0.01, "bits": 8})
    for g in grads:
        batch.micro_step(g)
    out = batch.apply().clone()
    opt = pipeline.AdamW(batch.ctx, y, 0.01, bits=8)
    opt.step(out)
    assert torch.equal(x, y) and int(batch.adamw.step_count) == 1
    x, y = x0.clone(), x0.clone()
    dist = pipeline.DistributedStep(table, W, "topk", optimizer={"kind": "adamw", "params": x, "lr": 0.01})
    out = dist.step(grads[0]).clone()
    pipeline.AdamW(dist.ctx, y, 0.01).step(out)
    assert torch.equal(x, y)


def test_unknown_optimisers_are_refused():
    table = _lm(64, 12)
    x = torch.zeros(table.stride, device="cuda")
    with pytest.raises(ValueError, match="kind"):
        pipeline.AccordionStep(table, 1, ("topk",), optimizer={"kind": "adam", "params": x, "lr": 0.1})
    with pytest.raises(ValueError, match="bits"):
        pipeline.AccordionStep(table, 1, ("topk",), optimizer={"kind": "adamw", "params": x, "lr": 0.1, "bits": 16})
    with pytest.raises(ValueError, match="one compressor"):
        pipeline.AccordionStep(table, 1, ("powersgd", "topk"), optimizer={"kind": "adamw", "params": x, "lr": 0.1})
    with pytest.raises(ValueError):
        pipeline.TokenEmbedding(binding.Context(table, 1), "no such layer", 4)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_large_clipped_step_replayed_as_a_graph(bits):
    """A table of more blocks than fit the GPU at once: norms, factor, coefficients and update, each launched behind the one
    before, give the same bits called one by one, in a captured graph, and with a synchronisation after every call."""
    table = wl.make_table(wl.shapes_vgg19bn(10))
    ctx = binding.Context(table, 1)
    g = torch.Generator(device="cuda").manual_seed(6)
    mask = torch.zeros(table.stride, device="cuda")
    for _, sl in table.slices():
        mask[sl] = 1.0
    x0 = torch.randn(table.stride, generator=g, device="cuda") * mask
    ds = [torch.randn(table.stride, generator=g, device="cuda") * mask for _ in range(3)]
    d = torch.empty_like(x0)

    def state(opt):
        s = [opt.m, opt.v] if bits == 32 else [t.view(torch.uint8) for t in (opt.m_code, opt.r_code, opt.m_scale, opt.r_scale)]
        return [opt.params, opt.step_count, opt.factor, opt.norm] + s

    runs = []
    for how in ("calls", "graph", "waits"):
        opt = pipeline.AdamW(ctx, x0.clone(), 1e-3, bits=bits, max_norm=1.0, seed=2)
        if how == "graph":
            d.copy_(ds[0])
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                launches = opt.step(d)
            assert launches == 5
        for src in ds:
            d.copy_(src)
            if how == "graph":
                graph.replay()
            elif how == "calls":
                opt.step(d)
            else:
                torch.cuda.synchronize()
                ctx.acc_layer_norms(d, 1, opt.norm2)
                torch.cuda.synchronize()
                ctx.acc_clip_factor(opt.norm2, 1.0, opt.factor, opt.norm)
                torch.cuda.synchronize()
                opt.max_norm = None
                f = opt.factor.clone()
                if bits == 32:
                    ctx.acc_adamw(d, opt.params, opt.m, opt.v, opt.step_count, opt.hyper, f)
                else:
                    ctx.acc_adamw_8bit(d, opt.params, opt.m_code, opt.r_code, opt.m_scale, opt.r_scale, opt.step_count,
                                       opt.hyper, 2, f)
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        runs.append([t.clone() for t in state(opt)])
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))
    assert int(runs[0][1]) == 3 and 0 < float(runs[0][2]) < 1


def test_embedding_calls_back_to_back_share_nothing_but_order():
    """Long and short calls on the same gradients, workspace and stream without a wait between them: the second
    touches nothing before the first is complete, though its kernels may be launched earlier."""
    table, W = _lm(3001, 24), 2
    ctx = binding.Context(table, W)
    g = torch.Generator(device="cuda").manual_seed(8)
    sets = [(_tokens(W, n, 3001, n), torch.randn(W, n, 24, generator=g, device="cuda")) for n in (9000, 40, 2500, 700)]
    ws = ctx.new_embedding_workspace(0, 9000)
    want = torch.zeros(W, table.stride, device="cuda")
    got = want.clone()
    for k, (tokens, dy) in enumerate(sets):
        ctx.acc_embedding_grad(0, tokens, dy, want, accumulate=k > 0, workspace=ws)
        torch.cuda.synchronize()
    for _ in range(5):
        for k, (tokens, dy) in enumerate(sets):
            ctx.acc_embedding_grad(0, tokens, dy, got, accumulate=k > 0, workspace=ws)
        out = got.clone()
        assert torch.equal(out, want)


@pytest.mark.parametrize("n", [40, 2500])
def test_calls_behind_copies_clears_and_other_streams(n):
    """Every call of a run, captured once and replayed, first behind a copy or a clear and behind torch's kernels that write
    its inputs, and with calls of two streams that meet: the bits of the same calls with a wait after each of them."""
    table, W, rows, cols = _lm(3001, 24), 2, 3001, 24
    ctx = [binding.Context(table, W) for _ in range(2)]  # (a context's workspace serves one stream at a time)
    g = torch.Generator(device="cuda").manual_seed(12)
    srcs = [(_tokens(W, n, rows, 30 + k), torch.randn(W, n, cols, generator=g, device="cuda")) for k in range(4)]
    tokens, dy = torch.empty_like(srcs[0][0]), torch.empty_like(srcs[0][1])
    x0 = torch.randn(table.stride, generator=g, device="cuda")
    ws = ctx[0].new_embedding_workspace(0, n)

    def state():
        z = lambda *shape: torch.zeros(*shape, device="cuda")
        return {"x": x0.clone(), "y": z(W, n, cols), "z": z(W, n, cols), "g": z(W, table.stride), "d": z(table.stride),
                "n2": torch.zeros(table.n_layers, dtype=torch.float64, device="cuda"), "f": z(1),
                "norm": torch.zeros(1, dtype=torch.float64, device="cuda")}

    def run(st, opt, other, wait):
        main = torch.cuda.current_stream()
        ctx[0].acc_embedding_lookup(0, st["x"], tokens, st["y"], 2.0)  # (behind a copy)
        wait()
        st["y"].add_(dy)
        wait()
        st["g"].zero_()
        wait()
        ctx[0].acc_embedding_grad(0, tokens, st["y"], st["g"], accumulate=True, workspace=ws)
        wait()
        torch.mean(st["g"], 0, out=st["d"])
        other.wait_stream(main)
        wait()
        with torch.cuda.stream(other):
            ctx[1].acc_layer_norms(st["d"], 1, st["n2"])
            ctx[1].acc_clip_factor(st["n2"], 0.5, st["f"], st["norm"])
        ctx[0].acc_embedding_lookup(0, st["x"], tokens, st["z"], 3.0)  # (reads what the update behind it changes)
        main.wait_stream(other)
        wait()
        ctx[0].acc_adamw(st["d"], st["x"], opt.m, opt.v, opt.step_count, opt.hyper, st["f"])
        wait()
        ctx[0].acc_embedding_lookup(0, st["x"], tokens, st["y"], 1.0)
        ctx[0].acc_embedding_grad(0, tokens, st["y"], st["g"], workspace=ws)
        wait()

    results = []
    for how in ("waits", "calls", "graph"):
        st, other = state(), torch.cuda.Stream()
        opt = pipeline.AdamW(ctx[0], st["x"], 1e-2)
        st["x"] = opt.params
        other.wait_stream(torch.cuda.current_stream())
        graph = None
        if how == "graph":
            tokens.copy_(srcs[0][0])
            dy.copy_(srcs[0][1])
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                run(st, opt, other, lambda: None)
        for tok, grad in srcs:
            dy.copy_(grad)
            tokens.copy_(tok)
            if graph is not None:
                graph.replay()
            else:
                run(st, opt, other, torch.cuda.synchronize if how == "waits" else lambda: None)
        torch.cuda.synchronize()
        cover = torch.zeros(table.stride, dtype=torch.bool, device="cuda")
        for _, sl in table.slices():
            cover[sl] = True
        results.append([st["x"][cover], st["g"][:, cover], st["y"], st["z"], st["n2"], st["f"], st["norm"], opt.step_count])
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    assert int(results[0][-1]) == 4 and ctx[0].acc_device_status() == 0


def test_a_call_into_a_broken_capture_fails_alone():
    """A launch that the runtime refuses (the stream's capture was invalidated by waiting for it) is an error of that call;
    the calls behind it, on streams in order, succeed."""
    rt = ctypes.CDLL("libcudart.so.12")
    table, W, n = _lm(), 2, 3000
    ctx = binding.Context(table, W)
    d = _grads(table, W, 1)
    opt = pipeline.AdamW(ctx, torch.zeros(table.stride, device="cuda"), 0.01)
    opt8 = pipeline.AdamW(ctx, torch.zeros(table.stride, device="cuda"), 0.01, bits=8)
    tokens, y = _tokens(W, n, 211, 2), torch.zeros(W, n, 26, device="cuda")
    emb = pipeline.TokenEmbedding(ctx, "encoder.weight", n)
    norm2 = torch.zeros(W, table.n_layers, dtype=torch.float64, device="cuda")
    side = torch.cuda.Stream()
    p = ctypes.c_void_p(side.cuda_stream)
    few = (tokens[:, :40].contiguous(), y[:, :40].contiguous())
    for call in (lambda s: ctx.acc_layer_norms(d, W, norm2, stream=s), lambda s: ctx.acc_clip_factor(opt.norm2, 1.0, opt.factor, stream=s),
                 lambda s: opt.step(d[0], s), lambda s: opt8.step(d[0], s), lambda s: emb.lookup(d[0], tokens, y, s),
                 lambda s: emb.backward(tokens, y, d, s), lambda s: emb.backward(*few, d, s)):
        torch.cuda.synchronize()
        call(None)
        torch.cuda.synchronize()
        assert rt.cudaStreamBeginCapture(p, 2) == 0  # (2: other threads and streams are not concerned)
        try:
            assert rt.cudaStreamSynchronize(p) != 0
            with pytest.raises(binding.AccError) as e:
                call(side)
        finally:
            graph = ctypes.c_void_p()
            assert rt.cudaStreamEndCapture(p, ctypes.byref(graph)) != 0
            rt.cudaGetLastError()
        assert e.value.status == 4
        call(None)
        call(side)
        torch.cuda.synchronize()
    assert ctx.acc_device_status() == 0
