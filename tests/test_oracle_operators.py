"""The float64 definitions that the GPU tests of the operators around the solves compare with, against autograd,
differences and properties that fix them."""
import numpy as np
import pytest
import torch

from oracle import operators as oo


@pytest.mark.parametrize("cols", [1, 31, 32, 33, 70])
def test_kept_values_are_within_half_a_step_and_keep_the_sign(cols):
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((50, cols)) * np.exp(3 * rng.standard_normal((50, 1)))
    q, s = oo.q8_pack(x)
    v = oo.q8_unpack(q, s, cols)
    step = np.repeat(np.ldexp(1.0, s.astype(int) - 127), 32, axis=1)[:, :cols]
    assert np.all(np.abs(v - x) <= step / 2) and np.all(v * x >= 0)
    assert np.all(q[:, cols:] == 0)
    # the smallest power of two that holds the block: half of it would not
    top = np.max(np.abs(np.pad(x, ((0, 0), (0, -cols % 32)))).reshape(50, -1, 32), axis=2)
    assert np.all(top < 127.5 * np.ldexp(1.0, s.astype(int) - 127))
    assert np.all(top >= 127.5 * np.ldexp(1.0, s.astype(int) - 128))
    # what is kept stays as it is
    q2, s2 = oo.q8_pack(v)
    assert np.array_equal(oo.q8_unpack(q2, s2, cols), v)


def test_kept_values_at_the_borders():
    x = np.zeros((9, 32))
    x[1, 3] = 127.5                        # 127.5 rounds past 127: the next power
    x[2, 3] = np.nextafter(np.float32(127.5), np.float32(0))
    x[3, 3], x[3, 4] = np.inf, 1.0
    x[4, 5] = np.nan
    x[5, :2] = 2.0 ** -149, -2.0 ** -126
    x[6, :4] = 64.0, 0.5, 1.5, -2.5        # step 1: ties to even
    x[7, 0] = 127.5 * 2.0 ** 121           # would round to 2^128
    x[8, 0] = np.nextafter(np.float32(x[7, 0]), np.float32(0))
    q, s = oo.q8_pack(x)
    assert list(s[:, 0]) == [1, 128, 127, 255, 255, 1, 127, 255, 248]
    assert q[1, 3] == 64 and q[2, 3] == 127 and not q[3].any() and not q[4].any()
    assert list(q[5, :2]) == [0, -1] and list(q[6, :4]) == [64, 0, 2, -2]
    v = oo.q8_unpack(q, s, 32)
    assert np.isnan(v[3]).all() and np.isnan(v[4]).all() and not v[0].any()


@pytest.mark.parametrize("gain", [True, False])
def test_norm_gradients_are_autograds_and_differences(gain):
    rng = np.random.default_rng(5)
    x, dy = rng.standard_normal((6, 9)) * 2 + 1, rng.standard_normal((6, 9))
    gamma, beta = (1 + 0.3 * rng.standard_normal(9), rng.standard_normal(9)) if gain else (np.ones(9), np.zeros(9))
    y, mean, rstd = oo.norm_forward(x, gamma, beta, 1e-3)
    dx, dg, db = oo.norm_backward(dy, x, gamma, mean, rstd)
    t = [torch.tensor(v, requires_grad=True) for v in (x, gamma, beta)]
    ty = torch.nn.functional.layer_norm(t[0], (9,), t[1], t[2], 1e-3)
    ty.backward(torch.tensor(dy))
    assert np.allclose(y, ty.detach().numpy(), atol=1e-13)
    for got, ref in zip((dx, dg, db), t):
        assert np.allclose(got, ref.grad.numpy(), atol=1e-12)
    loss = lambda a, g, b: float((oo.norm_forward(a, g, b, 1e-3)[0] * dy).sum())  # noqa: E731
    for k, got in enumerate((dx, dg, db)):
        args = [x, gamma, beta]
        d = rng.standard_normal(args[k].shape)
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + 1e-5 * d, args[k] - 1e-5 * d
        assert np.isclose((loss(*up) - loss(*down)) / 2e-5, (got * d).sum(), rtol=1e-7)


def test_weight_gradient_is_autograds():
    rng = np.random.default_rng(6)
    dy, x = rng.standard_normal((11, 4)), rng.standard_normal((11, 7))
    w, b = torch.zeros((4, 7), dtype=torch.float64, requires_grad=True), torch.zeros(4, dtype=torch.float64, requires_grad=True)
    (torch.tensor(x) @ w.T + b).backward(torch.tensor(dy))
    dW, db = oo.weight_grad(dy, x, 0.5)
    assert np.allclose(2 * dW, w.grad.numpy()) and np.allclose(2 * db, b.grad.numpy())
