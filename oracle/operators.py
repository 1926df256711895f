"""The operators around the layer solves in float64 numpy, from their definitions: rows kept in 8 bits, LayerNorm of rows
with its backward pass, the gradients of a linear map.  Shares no code with the library."""
import numpy as np

BLOCK = 32


def q8_pack(x):
    """x [rows, cols] -> (q int8 [rows, 32 * blocks], scale uint8 [rows, blocks])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    t = np.zeros((rows, blocks * BLOCK))
    t[:, :cols] = x
    t = t.reshape(rows, blocks, BLOCK)
    with np.errstate(invalid="ignore"):
        top = np.max(np.abs(t), axis=2)                   # NaN if there is one
    with np.errstate(invalid="ignore"):
        good = top < 127.5 * 2.0 ** 121
    top = np.where(good, top, 0.0)
    e = np.full(top.shape, -126)
    part, power = np.frexp(top)                           # top = part * 2^power, 1/2 <= part < 1, or 0
    e = np.maximum(e, np.where(top > 0, np.where(part * 128 < 127.5, power - 7, power - 6), -126))
    t = np.where(good[..., None], t, 0.0)
    q = np.rint(np.ldexp(t, -e[..., None]))               # ties to even
    assert np.all(np.abs(q) <= 127)
    return (q.astype(np.int8).reshape(rows, blocks * BLOCK), np.where(good, e + 127, 255).astype(np.uint8))


def q8_unpack(q, scale, cols):
    rows, blocks = scale.shape
    e = scale.astype(np.int64)
    v = np.ldexp(q.reshape(rows, blocks, BLOCK).astype(np.float64), (e - 127)[..., None])
    v = np.where((e == 255)[..., None], np.nan, v)
    return v.reshape(rows, blocks * BLOCK)[:, :cols]


def norm_forward(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        mean = x.mean(1)
        rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
        y = (x - mean[:, None]) * rstd[:, None] * gamma + beta
    return y, mean, rstd


def norm_backward(dy, x, gamma, mean, rstd):
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def weight_grad(dy, x, scale=1.0):
    return scale * (dy.T @ x), scale * dy.sum(0)
