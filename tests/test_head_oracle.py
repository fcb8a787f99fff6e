"""Pins of the head's oracle (CPU): closed forms, differences, library functions; and refusals of the calls that need no GPU."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as hor
from paper_2010_16248_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.lib()


def test_logprobs_equal_the_library_log_softmax_and_closed_forms():
    rng = np.random.default_rng(0)
    z = rng.normal(0, 3, (5, 11))
    z[2, 3:7] = -np.inf
    tokens = np.array([0, 10, 1, -1, 4])
    r = hor.token_logprobs(z, tokens, 0.7, 3)
    want = torch.log_softmax(torch.from_numpy(z) * 0.7, 1)
    for i in (0, 1, 2, 4):
        assert np.isclose(r["logp"][i], want[i, tokens[i]])
        p = want[i].exp()
        assert np.isclose(r["entropy"][i], torch.special.entr(p).sum())
        assert np.allclose(r["top_logp"][i], want[i].topk(3).values)
    assert r["logp"][3] == 0 and (r["top_index"][3] == -1).all()
    flat = hor.token_logprobs(np.full((1, 8), 2.5), [3], 1.0, 4)  # equal logits
    assert np.isclose(flat["entropy"][0], np.log(8)) and list(flat["top_index"][0]) == [0, 1, 2, 3]
    assert hor.token_logprobs(np.full((1, 4), -np.inf), [1], 1.0, 2)["logp"][0] == -np.inf


@pytest.mark.parametrize("scale", [1.0, 0.7, 1.5])
def test_gradient_equals_differences(scale):
    rng = np.random.default_rng(1)
    z = rng.normal(0, 2, (3, 9))
    z[1, 4] = -np.inf
    tokens, g, h = np.array([2, 0, 8]), rng.normal(size=3), rng.normal(size=3)

    def loss(z):
        r = hor.token_logprobs(z, tokens, scale, 0)
        return (g * r["logp"] + h * r["entropy"]).sum()

    r = hor.token_logprobs(z, tokens, scale, 0)
    got = hor.token_logprobs_grad(z, tokens, r["norm"], g, h, r["entropy"], scale)
    for i in range(3):
        for j in range(9):
            if z[i, j] == -np.inf:
                assert got[i, j] == 0
                continue
            a, b, eps = z.copy(), z.copy(), 1e-6
            a[i, j] += eps
            b[i, j] -= eps
            assert abs((loss(a) - loss(b)) / (2 * eps) - got[i, j]) < 1e-7


def test_checkpoint_codes_are_the_nearest_of_all_and_decode():
    rng = np.random.default_rng(2)
    x = rng.normal(0, 1, (7, 70)) * 10.0 ** rng.uniform(-6, 3, (7, 1))
    x[3, :32] = 0
    x[4, 5] = np.inf
    code, byte = hor.checkpoint_encode(x)
    assert code.shape == (7, 96) and byte.shape == (7, 3) and (code[:, 70:][np.arange(7) != 4] == 0).all()
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert byte[3, 0] == 0 and byte[4, 0] == 255
    for i in range(7):
        for j in range(70):
            if byte[i, j // 32] in (0, 255):
                continue
            s = 2.0 ** (float(byte[i, j // 32]) - 127)
            best = np.nanmin(np.abs(every * s - x[i, j]))
            assert abs(every[code[i, j]] * s - x[i, j]) == best
    top = np.abs(x[0, :32]).max() / 2.0 ** (float(byte[0, 0]) - 127)
    assert 128 <= top < 256
    values = hor.checkpoint_decode(code, byte, 70)
    fine = np.isfinite(values)
    assert np.array_equal(values[fine], (every[code[:, :70]] * np.repeat(2.0 ** (byte.astype(float) - 127), 32, 1)[:, :70])[fine])
    assert np.isnan(values[4, :32]).all()


def test_null_contexts_and_host_queries_are_refused(lib):
    assert lib.acc_token_logprobs(None, None, 0, 1, 5, 5, None, 0, 1.0, None, None, None, 0, None, None, None) == 1
    assert lib.acc_token_logprobs_grad(None, None, 0, 1, 5, 5, None, 0, 1.0, None, None, 0, None, 0, None, None, 0, 5, None) == 1
    assert lib.acc_checkpoint_store(None, None, 0, 1, 5, 5, None, 0, None, None, None) == 1
    assert lib.acc_checkpoint_load(None, None, None, 1, 5, None, 0, 5, None) == 1
    assert lib.acc_linear_grad_workspace_bytes(None, 0, 5, None) == 1
    assert lib.acc_linear_grad(None, 0, None, 0, 1, 5, 5, 1.0, None, None, None, 0, None, 0, None) == 1
    assert "vocabulary" in lib.acc_strerror(7).decode()
