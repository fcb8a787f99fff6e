"""The embedding's lookup and gradient against the fp64 oracle, through the C-ABI.

Tolerances.  Lookup: one fp32 product, rounded once more to bf16: equal to the same two roundings in torch, bit for bit.
Gradient: u = 2^-24.  A row with k tokens is a sum of k values in fp32, of at most k additions in all.  Up to 2048 tokens it
passes at most ceil(n / 32) additions of its half warp and the sums of at most 63 others (64 half warps that accumulate, 32
that overwrite); beyond that at most 16 of its warp and 7 of the other warps' sums in the first level, 32 and 7 in each level
above (128 chunks of the level below), each with an error of at most u times the
sum of the magnitudes; the scale is one fma more (2 u of the result with accumulation: the product is exact inside).
"""
import numpy as np
import pytest
import torch

from oracle import training_oracle as tor
from paper_2010_16248_b200 import binding, pipeline, workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _ctx(rows, cols, W, before=True):
    """The embedding as the middle layer of three, so that neighbours would show a stray write."""
    table = wl.make_table(([("v", (5,))] if before else []) + [("emb", (rows, cols)), ("after", (3, 7))])
    return table, binding.Context(table, W), table.names.index("emb")


def _slice(table, layer):
    o = int(table.offset[layer])
    return slice(o, o + int(table.rows[layer]) * int(table.cols[layer]))


def _tokens(rng, W, n, rows, kind, dtype=torch.int64):
    if kind == "zipf":
        t = np.minimum((rng.pareto(0.7, (W, n)) * 2).astype(np.int64), rows - 1)
        t = rng.permutation(rows)[t]
    elif kind == "same":
        t = np.full((W, n), rows - 1)
    elif kind == "padding":
        t = np.full((W, n), -1)
    else:
        t = rng.integers(0, rows, (W, n))
        if kind == "padded":
            t = np.where(rng.random((W, n)) < 0.3, -1 - rng.integers(0, 5, (W, n)), t)
    return torch.from_numpy(np.asarray(t)).to(dtype).cuda()


LOOKUPS = [(1, 1, 1), (2, 3, 5), (7, 8, 1), (50, 7, 33), (257, 64, 700), (3000, 650, 701), (41, 1030, 64), (5, 2, 0), (9, 4, 8),
           (70000, 5, 1000)]


@pytest.mark.parametrize("rows,cols,n", LOOKUPS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tok", [torch.int32, torch.int64])
def test_lookup(rows, cols, n, dtype, tok):
    rng = np.random.default_rng(rows + n)
    table, ctx, layer = _ctx(rows, cols, 1)
    g = torch.Generator(device="cuda").manual_seed(cols)
    params = torch.randn(table.stride, generator=g, device="cuda")
    tokens = _tokens(rng, 1, n, rows, "padded", tok)[0]
    out = torch.full((n, cols), 77.0, dtype=dtype, device="cuda")
    ctx.acc_embedding_lookup(layer, params, tokens, out, scale=1.7)
    emb = params[_slice(table, layer)].view(rows, cols)
    want = (emb[tokens.clamp(min=0).long()] * np.float32(1.7)).to(dtype)
    want[tokens < 0] = 0
    assert torch.equal(out, want)
    half_step = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8  # of the type; the scale itself was rounded to fp32
    exact = tor.embedding_lookup(emb.cpu().numpy(), tokens.cpu().numpy(), float(np.float32(1.7)))
    assert (np.abs(out.double().cpu().numpy() - exact) <= (half_step + 1.01 * U) * np.abs(exact)).all()
    assert ctx.last_launch_count() == (1 if n else 0) and ctx.acc_device_status() == 0


def _check_grad(table, ctx, layer, tokens, dy, grads0, grads, scale, accumulate):
    rows, cols = int(table.rows[layer]), int(table.cols[layer])
    sl = _slice(table, layer)
    W, n = tokens.shape
    levels = 0
    c = (n + 127) // 128
    while c > 1:
        c = (c + 127) // 128
        levels += 1
    most = (n + 31) // 32 + 63 if n <= 2048 else 23 + 39 * levels
    for w in range(W):
        t = tokens[w].cpu().numpy()
        y = dy[w].float().cpu().numpy()
        G, S, K = tor.embedding_grad(t, y, rows, float(np.float32(scale)))
        base = grads0[w, sl].double().cpu().numpy().reshape(rows, cols) if accumulate else 0.0
        want = base + G
        got = grads[w, sl].double().cpu().numpy().reshape(rows, cols)
        bound = 1.01 * U * (np.minimum(np.maximum(K - 1, 0), most)[:, None] * S + np.abs(G) + np.abs(want))
        bad = ~(np.abs(got - want) <= bound)
        assert not bad.any(), (w, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])
        if accumulate:  # rows without a token keep their bits
            still = K == 0
            assert np.array_equal(got[still], base[still])
        else:
            assert np.array_equal(got[K == 0], np.zeros_like(got[K == 0]))
    outside = torch.ones(grads.shape[1], dtype=torch.bool, device="cuda")
    outside[sl] = False
    assert torch.equal(grads[:, outside], grads0[:, outside])


def _run_grad(rows, cols, W, n, kind, dtype=torch.float32, tok=torch.int64, scale=1.0, accumulate=False, seed=0):
    rng = np.random.default_rng(seed + 31 * n + rows)
    table, ctx, layer = _ctx(rows, cols, W)
    g = torch.Generator(device="cuda").manual_seed(seed + n)
    tokens = _tokens(rng, W, n, rows, kind, tok)
    dy = torch.randn(W, n, cols, generator=g, device="cuda")
    dy = torch.where((tokens < 0)[..., None], float("nan"), dy).to(dtype)  # what lies at padding is not read
    grads0 = torch.randn(W, table.stride, generator=g, device="cuda")
    grads = grads0.clone()
    ws = ctx.new_embedding_workspace(layer, n)
    ws.random_(0, 256, generator=g)
    ctx.acc_embedding_grad(layer, tokens, dy, grads, scale=scale, accumulate=accumulate, workspace=ws)
    assert ctx.acc_device_status() == 0
    _check_grad(table, ctx, layer, tokens, dy, grads0, grads, scale, accumulate)
    again = grads0.clone()
    ws.random_(0, 256, generator=g)
    ctx.acc_embedding_grad(layer, tokens, dy, again, scale=scale, accumulate=accumulate, workspace=ws)
    assert torch.equal(grads, again)  # bit-reproducible, whatever the workspace held


@pytest.mark.parametrize("n", [0, 1, 2, 31, 32, 33, 63, 64, 65, 255, 256, 257, 700, 1025, 2047, 2048, 2049, 4097, 5000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad_lengths(n, accumulate):
    _run_grad(50, 6, 2, n, "padded", scale=2.5, accumulate=accumulate)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4), (2, 3), (300, 2), (257, 7), (256, 5), (255, 64), (65536, 3), (70000, 4),
                                       (33, 650), (20, 1030), (12, 513)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [37, 2500])
def test_grad_tables(rows, cols, dtype, n):
    _run_grad(rows, cols, 2, n, "uniform", dtype=dtype, tok=torch.int32, accumulate=n == 37)


@pytest.mark.parametrize("kind", ["zipf", "same", "padding"])
@pytest.mark.parametrize("n", [40, 1500, 40000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad_distributions(kind, n, accumulate):
    _run_grad(1000, 12, 3, n, kind, dtype=torch.bfloat16, scale=0.5, accumulate=accumulate)


def test_grad_layer_of_many_pieces_and_one_worker():
    _run_grad(40009, 13, 1, 900, "zipf")


def test_a_token_beyond_the_table_is_reported_and_reads_nothing():
    table, ctx, layer = _ctx(10, 6, 2)
    params = torch.randn(table.stride, device="cuda")
    for tok in (torch.int32, torch.int64):
        tokens = torch.tensor([[1, 10, 3], [2 ** 31 - 1, 0, 9]], dtype=tok, device="cuda")
        if tok == torch.int64:
            tokens[1, 0] = 2 ** 32 + 1  # must not be taken for row 1
        inside = torch.tensor([[True, False, True], [False, True, True]], device="cuda")
        out = torch.full((2, 3, 6), 5.0, device="cuda")
        ctx.acc_embedding_lookup(layer, params, tokens, out)
        assert ctx.acc_device_status() == binding.ACC_EINDEX
        ctx.acc_reset_device_status()
        want = params[_slice(table, layer)].view(10, 6)[torch.where(inside, tokens, 0).long()]
        assert torch.equal(out, torch.where(inside[..., None], want, 0.0))
        for n in (3, 2100):
            pad = torch.cat([tokens, torch.full((2, n - 3), -1, dtype=tok, device="cuda")], 1).contiguous()
            dy = torch.ones(2, n, 6, device="cuda")
            grads = torch.zeros(2, table.stride, device="cuda")
            ctx.acc_embedding_grad(layer, pad, dy, grads, workspace=ctx.new_embedding_workspace(layer, n))
            assert ctx.acc_device_status() == binding.ACC_EINDEX
            ctx.acc_reset_device_status()
            rows = grads[:, _slice(table, layer)].view(2, 10, 6).sum(2).cpu().numpy() / 6
            assert np.array_equal(rows, [[0, 1, 0, 1, 0, 0, 0, 0, 0, 0], [1, 0, 0, 0, 0, 0, 0, 0, 0, 1]])
    assert ctx.acc_device_status() == 0


def test_gradient_agrees_with_differences_of_the_lookup():
    """d/dE <dy, lookup(E)> by central differences in fp64 over the lookup's own fp32 outputs: the lookup is linear, so the
    difference over a step of 2^-3 is exact up to the roundings of the outputs (u times their size, over the step)."""
    rows, cols, n = 6, 4, 9
    table, ctx, layer = _ctx(rows, cols, 1)
    sl = _slice(table, layer)
    g = torch.Generator(device="cuda").manual_seed(0)
    params = torch.randn(table.stride, generator=g, device="cuda")
    tokens = torch.tensor([[0, 3, 3, 5, -1, 0, 3, 2, 2]], device="cuda")
    dy = torch.randn(1, n, cols, generator=g, device="cuda")
    grads = torch.zeros(1, table.stride, device="cuda")
    ctx.acc_embedding_grad(layer, tokens, dy, grads, scale=1.5, workspace=ctx.new_embedding_workspace(layer, n))
    out = torch.empty(1, n, cols, device="cuda")
    h = 2.0 ** -3
    for j in range(rows * cols):
        vals = []
        for sign in (1, -1):
            p = params.clone()
            p[sl.start + j] += sign * h
            ctx.acc_embedding_lookup(layer, p, tokens, out, scale=1.5)
            vals.append(float((out.double() * dy.double()).sum()))
        # 9 outputs of size < 10, each |dy| < 5, rounded parameters and products: 2 u a side
        assert abs((vals[0] - vals[1]) / (2 * h) - float(grads[0, sl.start + j])) < 9 * 10 * 5 * 4 * U / h


def test_streams_graphs_and_shared_buffers():
    """Two calls in flight on two streams with their own workspaces; a captured forward and backward pass, replayed on new
    tokens written into the same buffers."""
    rows, cols, W, n = 500, 10, 2, 3000
    table, ctx, layer = _ctx(rows, cols, W)
    rng = np.random.default_rng(1)
    g = torch.Generator(device="cuda").manual_seed(1)
    sets = [(_tokens(rng, W, n, rows, "zipf"), torch.randn(W, n, cols, generator=g, device="cuda")) for _ in range(2)]
    zero = torch.zeros(W, table.stride, device="cuda")
    want = []
    for tokens, dy in sets:
        out = zero.clone()
        ctx.acc_embedding_grad(layer, tokens, dy, out, workspace=ctx.new_embedding_workspace(layer, n))
        want.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    spaces = [ctx.new_embedding_workspace(layer, n) for _ in sets]
    outs = [zero.clone() for _ in sets]
    torch.cuda.synchronize()
    for s, ws, out, (tokens, dy) in zip(streams, spaces, outs, sets):
        ctx.acc_embedding_grad(layer, tokens, dy, out, workspace=ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    tokens, dy = sets[0][0].clone(), sets[0][1].clone()
    out = zero.clone()
    params = torch.randn(table.stride, generator=g, device="cuda")
    y = torch.zeros(W, n, cols, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.acc_embedding_lookup(layer, params, tokens, y)
        ctx.acc_embedding_grad(layer, tokens, dy, out, workspace=spaces[0])
    for k in (1, 0):
        tokens.copy_(sets[k][0])
        dy.copy_(sets[k][1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k])
        assert torch.equal(y, params[_slice(table, layer)].view(rows, cols)[tokens])


def test_refusals():
    table, ctx, layer = _ctx(10, 6, 2)
    lib = binding.lib()
    tokens = torch.zeros(2, 4, dtype=torch.int64, device="cuda")
    dy = torch.zeros(2, 4, 6, device="cuda")
    grads = torch.zeros(2, table.stride, device="cuda")
    ws = ctx.new_embedding_workspace(layer, 4)
    with pytest.raises(binding.AccError) as e:
        ctx.acc_embedding_grad(layer, tokens, dy, grads, workspace=None)
    assert e.value.status == 3
    with pytest.raises(binding.AccError) as e:
        ctx.acc_embedding_grad(layer, tokens, dy, grads, workspace=ws[:-256])
    assert e.value.status == 3
    with pytest.raises(binding.AccError) as e:
        ctx.acc_embedding_grad(layer, tokens, dy, grads, workspace=torch.zeros(ws.numel() + 256, dtype=torch.uint8, device="cuda")[16:])
    assert e.value.status == 2
    wide = torch.zeros(2 * 4 * 6 + 4, device="cuda")
    with pytest.raises(binding.AccError) as e:
        ctx.acc_embedding_grad(layer, tokens, wide[1:49].view(2, 4, 6), grads, workspace=ws)
    assert e.value.status == 2
    with pytest.raises(binding.AccError) as e:
        ctx.acc_embedding_lookup(layer, grads[0], tokens, wide[1:49].view(2, 4, 6))
    assert e.value.status == 2
    t, d, g, w = tokens.data_ptr(), dy.data_ptr(), grads.data_ptr(), ws.data_ptr()
    n, big = ws.numel(), 1 << 40
    assert lib.acc_embedding_grad(ctx._h, 0, t, 1, 4, 1.0, d, 0, g, 0, w, n, None) == 1           # a VECTOR layer
    assert lib.acc_embedding_grad(ctx._h, 3, t, 1, 4, 1.0, d, 0, g, 0, w, n, None) == 1           # no layer
    assert lib.acc_embedding_grad(ctx._h, -1, t, 1, 4, 1.0, d, 0, g, 0, w, n, None) == 1
    assert lib.acc_embedding_grad(ctx._h, layer, t, 2, 4, 1.0, d, 0, g, 0, w, n, None) == 1       # types
    assert lib.acc_embedding_grad(ctx._h, layer, t, 1, 4, 1.0, d, 2, g, 0, w, n, None) == 1
    assert lib.acc_embedding_grad(ctx._h, layer, t, 1, -1, 1.0, d, 0, g, 0, w, n, None) == 1      # lengths
    assert lib.acc_embedding_grad(ctx._h, layer, t, 1, (1 << 27) + 1, 1.0, d, 0, g, 0, w, big, None) == 1
    assert lib.acc_embedding_grad(ctx._h, layer, None, 1, 4, 1.0, d, 0, g, 0, w, n, None) == 1
    assert lib.acc_embedding_grad(ctx._h, layer, t + 4, 1, 4, 1.0, d, 0, g, 0, w, n, None) == 2
    assert lib.acc_embedding_lookup(ctx._h, layer, g, t, 1, (1 << 28) + 1, 1.0, d, 0, None) == 1
    assert lib.acc_embedding_lookup(ctx._h, layer, None, t, 1, 4, 1.0, d, 0, None) == 1


@pytest.mark.parametrize("n", [131072 - 1, 131072 + 1, 200000])
def test_grad_many_sort_tiles(n):
    """Either side of the count of tiles from which the sort's counts are summed by a kernel of their own."""
    _run_grad(700, 8, 1, n, "zipf", dtype=torch.bfloat16)


@pytest.mark.parametrize("rows,n", [((1 << 21) - 1, 900), ((1 << 21) - 1, 2048), (1 << 21, 900), (1 << 21, 2048), ((1 << 21) + 1, 900), ((1 << 24) + 3, 2100)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad_tables_of_many_rows(rows, n, accumulate):
    """Rows that just fit, or no longer fit, a word beside the position; rows of more than three digits."""
    cols = 2
    table, ctx, layer = _ctx(rows, cols, 1)
    rng = np.random.default_rng(n)
    t = rng.integers(0, rows, (1, n))
    t[0, ::7] = t[0, -1] = rows - 1
    tokens = torch.from_numpy(t).cuda()
    dy = torch.randn(1, n, cols, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda")
    grads = torch.ones(1, table.stride, device="cuda")
    ctx.acc_embedding_grad(layer, tokens, dy, grads, accumulate=accumulate, workspace=ctx.new_embedding_workspace(layer, n))
    exact = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    exact.index_put_((tokens[0],), dy[0].double(), accumulate=True)
    size = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    size.index_put_((tokens[0],), dy[0].double().abs(), accumulate=True)
    got = grads[0, _slice(table, layer)].view(rows, cols).double()
    base = 1.0 if accumulate else 0.0
    # at most 127 additions a row (64 + 63, or 16 + 7 and 32 + 7), the scale's fma
    bound = 1.01 * U * (127 * size + (exact + base).abs() + exact.abs())
    assert bool(((got - base - exact).abs() <= bound).all())
    outside = torch.ones(table.stride, dtype=torch.bool, device="cuda")
    outside[_slice(table, layer)] = False
    assert bool((grads[0, outside] == 1.0).all())


def test_offsets_beyond_32_bits():
    """The second worker's layer lies behind element 2^31 of the gradient buffers, the table behind element 2^31 of the
    parameters."""
    off, rows, cols, n = 2 ** 31 + 2 ** 18, 50, 6, 90
    stride = off + 1024
    table = wl.LayerTable(["far"], np.array([off], np.int64), np.array([rows], np.int32), np.array([cols], np.int32),
                          np.array([wl.MATRIX], np.int32), stride)
    ctx = binding.Context(table, 2)
    g = torch.Generator(device="cuda").manual_seed(2)
    params = torch.empty(stride, device="cuda")
    emb = torch.randn(rows, cols, generator=g, device="cuda")
    params[off:off + rows * cols] = emb.reshape(-1)
    grads = torch.empty(2, stride, device="cuda")
    grads[:, off:].fill_(3.0)
    for length in (n, 2500):
        tokens = _tokens(np.random.default_rng(3), 2, length, rows, "padded")
        out = torch.empty(2, length, cols, device="cuda")
        ctx.acc_embedding_lookup(0, params, tokens, out)
        want = emb[tokens.clamp(min=0)]
        want[tokens < 0] = 0
        assert torch.equal(out, want)
        ctx.acc_embedding_grad(0, tokens, out, grads, workspace=ctx.new_embedding_workspace(0, length))
        for w in range(2):
            G, S, K = tor.embedding_grad(tokens[w].cpu().numpy(), out[w].cpu().numpy(), rows, 1.0)
            got = grads[w, off:off + rows * cols].view(rows, cols).double().cpu().numpy()
            assert (np.abs(got - G) <= 1.01 * U * (np.minimum(np.maximum(K - 1, 0), 127)[:, None] * S + 2 * np.abs(G))).all()
        assert bool((grads[:, off + rows * cols:] == 3.0).all())


@pytest.mark.parametrize("rows,cols,n", [((1 << 21) + 1, 2, 900), (1 << 21, 3, 900), (3, (1 << 20) + 4, 5)])
def test_an_empty_batch_on_a_large_table(rows, cols, n):
    """No tokens, on tables too large for the one launch of few tokens: one launch clears the layer behind whatever ran
    before it, and the calls behind it (a gradient that is added, norms, clip and update) find it cleared: the bits of the
    same calls with a wait after each, and of the gradient written at once."""
    W = 2
    table, ctx, layer = _ctx(rows, cols, W)
    sl = _slice(table, layer)
    g = torch.Generator(device="cuda").manual_seed(n)
    tokens = _tokens(np.random.default_rng(rows), W, n, rows, "uniform")
    dy = torch.randn(W, n, cols, generator=g, device="cuda")
    none, nothing = tokens[:, :0].contiguous(), dy[:, :0].contiguous()
    ws = ctx.new_embedding_workspace(layer, n)
    x0 = torch.randn(table.stride, generator=g, device="cuda")
    want = torch.ones(W, table.stride, device="cuda")
    ctx.acc_embedding_grad(layer, tokens, dy, want, scale=0.5, workspace=ws)
    runs = []
    for waits in (True, False, False, False):
        wait = torch.cuda.synchronize if waits else lambda: None
        opt = pipeline.AdamW(ctx, x0.clone(), 1e-2, max_norm=0.5)
        grads = torch.full((W, table.stride), 1.0, device="cuda")
        torch.cuda.synchronize()
        ctx.acc_embedding_grad(layer, tokens, dy, grads, scale=3.0, workspace=ws)
        wait()
        ctx.acc_embedding_grad(layer, none, nothing, grads, workspace=ws)
        assert ctx.last_launch_count() == 1
        wait()
        ctx.acc_embedding_grad(layer, tokens, dy, grads, scale=0.5, accumulate=True, workspace=ws)
        wait()
        opt.step(grads[0])
        wait()
        added = grads.clone()
        ctx.acc_embedding_grad(layer, none, nothing, grads, workspace=ws)
        opt.step(grads[1])
        torch.cuda.synchronize()
        assert torch.equal(added, want)
        assert not bool(grads[:, sl].any()) and bool((grads[:, :sl.start] == 1.0).all()) and bool((grads[:, sl.stop:] == 1.0).all())
        ctx.acc_embedding_grad(layer, none, nothing, grads, accumulate=True, workspace=ws)
        assert ctx.last_launch_count() == 0
        runs.append([opt.params, opt.m, opt.v, opt.norm, opt.step_count])
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))
    assert ctx.acc_device_status() == 0


@pytest.mark.parametrize("W", [1, 3])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad_many_sort_tiles_of_several_workers(W, accumulate):
    """Sort counts summed by a kernel of their own, for every worker, written and added."""
    _run_grad(700, 6, W, 131072 + 2049, "padded", dtype=torch.bfloat16, tok=torch.int32, scale=0.5, accumulate=accumulate)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad_of_more_than_three_levels(dtype, accumulate):
    """2 * 128^3 + 300 tokens per worker: partial sums of the third level go where those of the first were.  Rows of a fraction
    of all tokens, so that runs cross the edges of every level's chunks; the second worker's batch is padded.  All values are
    positive: a lost or repeated partial sum would be off by far more than the bound, whose 140 additions are those of four levels."""
    rows, cols, W, n = 7, 2, 2, 2 * 128 ** 3 + 300
    table, ctx, layer = _ctx(rows, cols, W)
    sl = _slice(table, layer)
    g = torch.Generator(device="cuda").manual_seed(5)
    share = torch.tensor([0.1, 0.6, 0.05, 1e-5, 0.1, 0.05, 0.1], device="cuda")
    tokens = torch.multinomial(share, W * n, replacement=True, generator=g).view(W, n)
    tokens[1] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.01, -1, tokens[1])
    dy = (torch.rand(W, n, cols, generator=g, device="cuda") + 0.5).to(dtype)
    grads = torch.rand(W, table.stride, generator=g, device="cuda")
    before = grads.clone()
    ctx.acc_embedding_grad(layer, tokens, dy, grads, scale=0.5, accumulate=accumulate, workspace=ctx.new_embedding_workspace(layer, n))
    assert ctx.acc_device_status() == 0
    for w in range(W):
        live = tokens[w] >= 0
        exact = torch.zeros(rows, cols, dtype=torch.float64, device="cuda").index_add_(0, tokens[w][live], 0.5 * dy[w][live].double())
        want = exact + (before[w, sl].view(rows, cols).double() if accumulate else 0.0)
        got = grads[w, sl].view(rows, cols).double()
        # (u of every addition's result, at most the whole sum; the fp64 sums' own error is 2^-53 n of it, far less)
        assert bool(((got - want).abs() <= 1.01 * U * (140 * exact + exact + want)).all())
    outside = torch.ones(table.stride, dtype=torch.bool, device="cuda")
    outside[sl] = False
    assert torch.equal(grads[:, outside], before[:, outside])
