"""The oracle of the AdamW step and its 8-bit states (no GPU needed)."""
import numpy as np
import pytest
import torch

import oracle.step_oracle as O


def test_a_step_is_torchs():
    g = np.random.default_rng(0)
    p, m, v = torch.tensor(g.normal(size=50)), np.zeros(50), np.zeros(50)
    q = torch.nn.Parameter(p.clone())
    opt = torch.optim.AdamW([q], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    x = p.numpy().copy()
    for t in range(1, 6):
        grad = g.normal(size=50)
        q.grad = torch.tensor(grad)
        opt.step()
        x, m, v = O.adamw(x, grad, m, v, t, 0.01, (0.8, 0.95), 1e-6, 0.1)
        assert np.allclose(x, q.detach().numpy(), rtol=0, atol=1e-14)


@pytest.mark.parametrize("fmt,dtype", [(O.M_FORMAT, torch.float8_e4m3fn), (O.V_FORMAT, torch.float8_e5m2)])
def test_codes_are_the_formats(fmt, dtype):
    mantissa, bias, top = fmt
    last = 0x7E if top == 8 else 0x7B
    all_codes = np.arange(last + 1)
    values = torch.arange(last + 1, dtype=torch.uint8).view(dtype).double().numpy()
    assert np.array_equal(O.value(all_codes, mantissa, bias), values) and values[-1] == 1.75 * 2.0 ** top
    for r in (0, 65535):                                          # what a code holds exactly is never rounded
        assert np.array_equal(O.codes(values, r, mantissa, bias), all_codes)
    between = 0.75 * values[:-1] + 0.25 * values[1:]
    for r, up in ((0, 0), (49151, 0), (49152, 1), (65535, 1)):
        assert np.array_equal(O.codes(between, r, mantissa, bias), all_codes[:-1] + up), r


def test_scales():
    x = np.zeros(600)
    x[5], x[300], x[520] = 448.0, -449.0, 1e-45
    assert list(O.scales(x, 8)) == [1.0, 2.0, 2.0 ** -126]


def test_words_are_a_permutation_and_differ_by_tensor_and_step():
    at = np.arange(1 << 16)
    a = O.words(at, 1, 1, 0)
    assert len(np.unique(a)) == len(at)
    assert abs(a.mean() / 2 ** 32 - 0.5) < 0.01 and abs((a & np.uint64(0xFFFF)).mean() / 65536 - 0.5) < 0.01
    for other in (O.words(at, 2, 1, 0), O.words(at, 1, 2, 0), O.words(at, 1, 1, 1), O.words(at + 2 ** 32, 1, 1, 0)):
        assert np.mean(a == other) < 0.001
