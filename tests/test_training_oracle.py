"""CPU pins of oracle/training_oracle.py (against torch's own AdamW and autograd, closed forms and exhaustive checks of the
8-bit format), and the refusals of the training operators that need no GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import training_oracle as tor
from paper_2010_16248_b200 import binding, build, workloads as wl
from tests import helpers as H
from tests.test_host_abi import _hostless_context


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.lib()


# ---- oracle pins -------------------------------------------------------------------------------------------------- #
def test_adamw_is_torchs():
    rng = np.random.default_rng(0)
    x0 = rng.standard_normal(40)
    p = torch.nn.Parameter(torch.tensor(x0, dtype=torch.float64))
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.9, 0.99), eps=1e-7, weight_decay=0.1)
    x, m, v, step = x0.copy(), np.zeros(40), np.zeros(40), 0
    for _ in range(7):
        g = rng.standard_normal(40)
        p.grad = torch.tensor(g)
        opt.step()
        x, m, v, step = tor.adamw(g, x, m, v, step, (0.01, 0.9, 0.99, 1e-7, 0.1), [(0, 4, 10, 0)])
        np.testing.assert_allclose(x, p.detach().numpy(), rtol=1e-13, atol=1e-15)
    assert step == 7


def test_adamw_decay_of_vectors_padding_and_skipped_steps():
    layers = [(0, 1, 3, 1), (4, 2, 2, 0)]
    x = np.ones(12)
    z = np.zeros(12)
    y, *_ = tor.adamw(z, x, z, z, 0, (0.5, 0.9, 0.9, 1e-8, 0.1), layers, decay_vectors=False)
    assert np.array_equal(y, [1, 1, 1, 1, .95, .95, .95, .95, 1, 1, 1, 1])
    y, _, _, t = tor.adamw(z, x, z, z, 5, (0.5, 0.9, 0.9, 1e-8, 0.1), layers, factor=np.nan)
    assert t == 5 and np.array_equal(y, x)


def test_clip_factor():
    assert tor.clip_factor([9.0, 16.0], 2.5) == (0.5, 5.0)
    assert tor.clip_factor([9.0, 16.0], 7.0)[0] == 1.0
    assert np.isnan(tor.clip_factor([9.0, np.inf], 7.0)[0])
    assert tor.clip_factor([0.0], 0.0)[0] == 1.0


def test_e4m3_values_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(tor.e4m3_values(), want)
    np.testing.assert_array_equal(tor.scale_values()[:255], codes.view(torch.float8_e8m0fnu).double().numpy()[:255])


def test_encode_is_unbiased_and_hits_the_neighbours():
    """Over all 2^16 random words the mean of the two neighbouring codes is the value, up to the words' own resolution;
    values on the grid stay."""
    val = tor.e4m3_values()
    rnd = np.arange(65536)
    for y in (200.0, 130.7, 255.9, 128.0, 1.0, 0.3333, 2.0 ** -6, 0.01, 2.0 ** -9, 1e-3, 1e-5):
        x = np.array([255.0] + [y] * 65536) if y < 128 else np.full(65537, y)
        byte, code, _ = tor.encode_block(x, np.concatenate([[0], rnd]), tor.LOWEST_M, False)
        assert byte == 127
        got = val[code[1:]]
        grid = 2.0 ** (max(np.floor(np.log2(y)), -6) - 3)
        assert len(np.unique(got)) <= 2 and np.all(np.abs(got - y) < grid * (1 + 2 ** -16))
        assert abs(got.mean() - y) <= grid * 2.0 ** -16
    byte, code, _ = tor.encode_block(np.array([200.0, 1e-9, 0.0, -0.0]), np.zeros(4), tor.LOWEST_R, True)
    assert list(code[1:]) == [1, 0, 128]
    assert tor.encode_block(np.array([1.0, np.nan]), np.zeros(2), tor.LOWEST_R, True)[0] == 255


def test_random_words_are_spread():
    w = tor.random_words(3, 17, np.arange(1 << 16))
    assert len(np.unique(w)) == 1 << 16                       # a bijection of the element
    for half in (w & np.uint64(0xFFFF), w >> np.uint64(16)):  # mean of n uniform values: standard error 1/sqrt(12 n)
        assert abs(half.astype(np.float64).mean() / 65536 - 0.5) < 5 / np.sqrt(12 * 65536)
    assert np.mean(w == tor.random_words(3, 18, np.arange(1 << 16))) < 1e-3


def test_embedding_is_autograds():
    rng = np.random.default_rng(2)
    table = rng.standard_normal((7, 5))
    tokens = np.array([3, 0, 3, 6, -1, 3, 9])
    keep = (tokens >= 0) & (tokens < 7)
    p = torch.tensor(table, requires_grad=True)
    y = torch.nn.functional.embedding(torch.tensor(np.where(keep, tokens, 0)), p) * 2.5 * torch.tensor(keep)[:, None]
    dy = rng.standard_normal((7, 5))
    y.backward(torch.tensor(dy))
    np.testing.assert_allclose(tor.embedding_lookup(table, tokens, 2.5), y.detach().numpy())
    G, S, K = tor.embedding_grad(tokens, dy, 7, 2.5)
    np.testing.assert_allclose(G, p.grad.numpy())
    assert list(K) == [1, 0, 0, 3, 0, 0, 1] and np.all(S >= np.abs(G) - 1e-15)


# ---- refusals that need no GPU ------------------------------------------------------------------------------------ #
def test_null_and_unknown_arguments_are_refused(lib):
    n = C.c_size_t()
    assert lib.acc_adamw(None, 16, 16, 16, 16, 16, 16, None, None, 0, None) == 1
    assert lib.acc_adamw_8bit(None, 16, 16, 16, 16, 16, 16, 16, 16, None, None, 0, 0, None) == 1
    assert lib.acc_clip_factor(None, 16, 1.0, 16, None, None) == 1
    assert lib.acc_adamw_layout(None, None, None) == 1
    assert lib.acc_embedding_lookup(None, 0, 16, 16, 0, 1, 1.0, 16, 0, None) == 1
    assert lib.acc_embedding_grad(None, 0, 16, 0, 1, 1.0, 16, 0, 16, 0, 256, 1 << 20, None) == 1
    assert lib.acc_embedding_workspace_bytes(None, 0, 1, C.byref(n)) == 1
    assert lib.acc_strerror(binding.ACC_EINDEX).decode().startswith("a token id")


def _context(W=2):
    table = wl.make_table([("a", (6, 10)), ("v", (5,)), ("b", (4, 8))])
    c = _hostless_context(table, W)
    c.q_row = np.where(table.kind == wl.MATRIX, np.arange(3), -1)
    c.adamw_blocks = len(tor.block_starts(H.layers_of(table)))
    return c, table.stride


def test_binding_checks_the_adamw_tensors():
    c, S = _context()
    f = lambda n: torch.zeros(n)                                   # noqa: E731
    step, hyper = torch.zeros(1, dtype=torch.int64), torch.zeros(5, dtype=torch.float64)
    ok = dict(d=f(S), params=f(S), m=f(S), v=f(S), step=step, hyper=hyper)
    for name in ok:
        with pytest.raises(ValueError, match=name):
            c.acc_adamw(**{**ok, name: ok[name][:-1].clone()})
    with pytest.raises(ValueError, match="hyper.*dtype"):
        c.acc_adamw(**{**ok, "hyper": f(5)})
    with pytest.raises(ValueError, match="params_bf16"):
        c.acc_adamw(**ok, params_bf16=f(S))
    with pytest.raises(ValueError, match="grad_scale"):
        c.acc_adamw(**ok, grad_scale=f(0))
    with pytest.raises(ValueError, match="CUDA"):
        c.acc_adamw(**ok)
    c8 = lambda n: torch.zeros(n, dtype=torch.uint8).view(torch.float8_e4m3fn)   # noqa: E731
    s8 = lambda n: torch.zeros(n, dtype=torch.uint8).view(torch.float8_e8m0fnu)  # noqa: E731
    ok = dict(d=f(S), params=f(S), m_code=c8(S), r_code=c8(S), m_scale=s8(c.adamw_blocks), r_scale=s8(c.adamw_blocks),
              step=step, hyper=hyper)
    for name in ok:
        with pytest.raises(ValueError, match=name):
            c.acc_adamw_8bit(**{**ok, name: ok[name][:-1].clone()})
    with pytest.raises(ValueError, match="r_code.*dtype"):
        c.acc_adamw_8bit(**{**ok, "r_code": torch.zeros(S, dtype=torch.uint8)})
    with pytest.raises(ValueError, match="CUDA"):
        c.acc_adamw_8bit(**ok)
    with pytest.raises(ValueError, match="norm2_layers"):
        c.acc_clip_factor(torch.zeros(2, dtype=torch.float64), 1.0, f(1))
    with pytest.raises(ValueError, match="factor"):
        c.acc_clip_factor(torch.zeros(3, dtype=torch.float64), 1.0, f(0))


def test_binding_checks_the_embedding_tensors():
    W = 2
    c, S = _context(W)
    f = lambda *n: torch.zeros(*n)                                 # noqa: E731
    tok = torch.zeros(W, 3, dtype=torch.int64)
    with pytest.raises(ValueError, match="MATRIX"):
        c.acc_embedding_lookup(1, f(S), tok, f(W, 3, 5))
    with pytest.raises(ValueError, match="MATRIX"):
        c.acc_embedding_lookup(3, f(S), tok, f(W, 3, 5))
    with pytest.raises(ValueError, match="tokens"):
        c.acc_embedding_lookup(0, f(S), tok.to(torch.int16), f(W, 3, 10))
    with pytest.raises(ValueError, match="out"):
        c.acc_embedding_lookup(0, f(S), tok, f(W, 3, 9))
    with pytest.raises(ValueError, match="out"):
        c.acc_embedding_lookup(0, f(S), tok, f(W, 3, 10).half())
    with pytest.raises(ValueError, match="params"):
        c.acc_embedding_lookup(0, f(c.extent - 1), tok, f(W, 3, 10))
    with pytest.raises(ValueError, match="contiguous"):
        c.acc_embedding_lookup(0, f(S), tok.t(), f(W, 3, 10))
    with pytest.raises(ValueError, match="CUDA"):
        c.acc_embedding_lookup(0, f(S), tok, f(W, 3, 10))
    ws = torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match="tokens"):
        c.acc_embedding_grad(0, tok[:, :2].reshape(-1)[:3].clone(), f(3, 10), f(W, S), workspace=ws)
    with pytest.raises(ValueError, match="tokens"):
        c.acc_embedding_grad(0, tok.reshape(3, 2), f(3, 2, 10), f(W, S), workspace=ws)
    with pytest.raises(ValueError, match="dy"):
        c.acc_embedding_grad(0, tok, f(W, 2, 10), f(W, S), workspace=ws)
    with pytest.raises(ValueError, match="grads"):
        c.acc_embedding_grad(0, tok, f(W, 3, 10), f(S), workspace=ws)
    with pytest.raises(ValueError, match="CUDA"):
        c.acc_embedding_grad(0, tok, f(W, 3, 10), f(W, S), workspace=ws)
