"""The float64 definitions of oracle/logits.py against torch's own log_softmax with autograd, and the gradients' formulas
against differences of the values."""
import numpy as np
import pytest
import torch

from oracle import logits as ol


def draw(rows=7, cols=23, kept=5, seed=0):
    rng = np.random.default_rng(seed)
    z = 2.0 * rng.standard_normal((rows, cols))
    tokens = rng.integers(0, cols, rows)
    tokens[2] = -1
    ids = np.stack([rng.permutation(cols)[:kept] for _ in range(rows)])
    ids[1, 3:], ids[4], ids[5, 1] = -1, -1, ids[5, 0]
    return z, tokens, ids, rng.standard_normal((rows, kept)), rng.standard_normal(rows), rng.standard_normal(rows)


@pytest.mark.parametrize("tau", [1.0, 0.7, 3.0])
def test_against_autograd(tau):
    z, tokens, ids, y, g, h = draw()
    zt = torch.tensor(z, requires_grad=True)
    lp = torch.log_softmax(zt / tau, 1)
    some = torch.tensor(tokens >= 0)
    logprob = torch.where(some, lp.gather(1, torch.tensor(tokens).clamp(min=0)[:, None])[:, 0], 0.0)
    entropy = -(lp.exp() * lp).sum(1)
    (logprob @ torch.tensor(g) + entropy @ torch.tensor(h)).backward()
    a, b, c = ol.logprobs(z, tokens, tau)
    for got, ref in ((a, logprob), (b, entropy), (c, torch.logsumexp(zt / tau, 1)), (ol.logprobs_gradient(z, tokens, g, h, tau), zt.grad)):
        assert np.allclose(got, ref.detach().numpy(), rtol=1e-12, atol=1e-13)
    zt.grad = None
    live = torch.tensor(ids >= 0)
    q = torch.softmax(torch.where(live, torch.tensor(y) / tau, -1e300), 1) * live
    lp = torch.log_softmax(zt / tau, 1)
    loss = (torch.xlogy(q, q) - q * lp.gather(1, torch.tensor(ids).clamp(min=0))).sum(1)
    (loss @ torch.tensor(g)).backward()
    got, _ = ol.distill(z, ids, y, tau)
    assert np.allclose(got, loss.detach().numpy(), rtol=1e-12, atol=1e-13) and got[4] == 0
    assert np.allclose(ol.distill_gradient(z, ids, y, g, tau), zt.grad.numpy(), rtol=1e-12, atol=1e-13)


@pytest.mark.parametrize("truncated", [False, True])
def test_gradients_against_differences(truncated):
    z, tokens, ids, y, g, h = draw(6, 6, 3, 1)
    tau, step = 1.3, 1e-5
    lse = np.log(np.exp(y / tau).sum(1)) + 0.4 if truncated else None

    def one(z):
        lp, H, _ = ol.logprobs(z, tokens, tau)
        return lp @ g + H @ h

    def two(z):
        return ol.distill(z, ids, y, tau, lse)[0] @ g
    for f, d in ((one, ol.logprobs_gradient(z, tokens, g, h, tau)), (two, ol.distill_gradient(z, ids, y, g, tau, lse))):
        for r in range(z.shape[0]):
            for i in range(z.shape[1]):
                e = np.zeros_like(z)
                e[r, i] = step
                # central differences err by step^2 / 6 of the third derivative (below 10 here) and by rounding, 1e-15 / step
                assert abs((f(z + e) - f(z - e)) / (2 * step) - d[r, i]) < 1e-9


def test_largest_by_value_then_id():
    z = np.array([[1.0, 3.0, 3.0, 2.0, -0.0, 0.0], [5.0, -np.inf, 5.0, 5.0, -np.inf, 5.0]])
    assert ol.largest(z, 6).tolist() == [[1, 2, 3, 0, 4, 5], [0, 2, 3, 5, 1, 4]]


def test_rows_without_a_distribution():
    z = np.zeros((5, 4))
    z[1], z[2, 1], z[3, 2], z[4, 0] = -np.inf, np.nan, np.inf, -np.inf
    lp, H, lse = ol.logprobs(z, [0, 1, 1, -1, 0])
    assert lp[1] == lse[1] == -np.inf and H[1] == 0 and np.isnan(lp[2]) and np.isnan(H[2]) and np.isnan(lse[3]) and lp[3] == 0
    assert lp[4] == -np.inf and np.isclose(H[4], np.log(3))
    d = ol.logprobs_gradient(z, [0, 1, 1, -1, 4], np.ones(5))
    assert (d[1] == 0).all() and np.isnan(d[2]).all() and (d[3] == 0).all() and np.isnan(d[4]).all()
    ids = np.array([[-1, -1], [0, 1], [0, 1], [1, 4], [0, 1]])
    loss, _ = ol.distill(z, ids, np.array([[0.0, 0], [0, 0], [0, 0], [0, 0], [-np.inf, 0]]))
    assert loss[0] == 0 and loss[1] == np.inf and np.isnan(loss[2]) and np.isnan(loss[3]) and np.isclose(loss[4], np.log(3))


def test_teachers_beyond_the_range():
    """With a log-sum-exp a share may be any number: those that 32 bits do not hold, alone or summed up, are none."""
    inf, nan = np.inf, np.nan
    ids = np.array([[0, 1]] * 8 + [[0, -1]])
    y = np.array([[0.0, 0], [inf, 0], [200, 0], [88.5, 88.5], [0, 0], [0, 0], [0, 0], [-inf, -inf], [0, inf]])
    lse = np.array([0.5, 0, 0, 0, -inf, inf, nan, 0, 0.5])
    q = ol.teacher(ids, y, 1.0, lse, 4)
    assert np.isnan(q).all(1).tolist() == [False, True, True, True, True, False, True, False, False]
    assert np.allclose(q[0], np.exp(-0.5)) and (q[5] == 0).all() and (q[7] == 0).all() and np.allclose(q[8], [np.exp(-0.5), 0])
    loss, _ = ol.distill(np.zeros((9, 4)), ids, y, 1.0, lse)
    d = ol.distill_gradient(np.zeros((9, 4)), ids, y, None, 1.0, lse)
    assert (np.isnan(loss) == np.isnan(q).any(1)).all() and (np.isnan(d).all(1) == np.isnan(q).any(1)).all() and (d[5] == 0).all()
