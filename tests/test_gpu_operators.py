"""The operators around the solves on the GPU against their float64 definitions (oracle/operators.py): 8-bit rows bit for
bit, LayerNorm of rows and the gradients from kept rows within bounds that follow from the arithmetic.

u = 2^-24 is half a step of fp32, relative; sums that are taken in fp32 err by at most (additions in sequence) * u * (sum
of magnitudes); an output of fewer bits adds half of its step."""
import threading
import types

import numpy as np
import pytest
import torch

from oracle import operators as oo
from paper_2601_09026_amd import binding as mb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16
WIDTHS = [1, 2, 3, 4, 5, 7, 31, 32, 33, 64, 65, 100, 128, 130, 255, 256, 260, 385, 512, 515, 768, 769, 1000, 1024, 1026, 2048,
          2051, 4096, 4100, 8192, 8200, 16383, 16384]


def say(*a):
    print("[case]", *a, flush=True)


def rand(seed, *shape, spread=1.0, offset=0.0, dtype=F32):
    rng = np.random.default_rng(seed)
    return torch.from_numpy((rng.standard_normal(shape) * spread + offset).astype(np.float32)).to(dtype).cuda()


def wide(t, pad, at=1):
    """The same rows as a slice of wider ones, starting `at` elements into them; the rest is NaN."""
    big = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    view = big[:, at:at + t.shape[1]]
    view.copy_(t)
    return big, view


def n64(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, bound, what):
    got = n64(got)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= bound + 1e-300)          # NaN fails
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - ref) / (bound + 1e-300)):.3g} times the bound"


def kept(t):
    """8-bit rows of a device tensor by the definition."""
    q, s = oo.q8_pack(n64(t))
    return mb.Q8Rows(torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), t.shape[1])


def same_rows(got, ref):
    assert torch.equal(got.scale, ref.scale) and torch.equal(got.q, ref.q)


# ------------------------------------------------------------------ 8-bit rows
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_pack_and_unpack(cols, dtype):
    say("pack", cols, dtype)
    for rows in (1, 3, 130):
        rng = np.random.default_rng(cols)
        x = torch.from_numpy((rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-40, 40, (rows, cols)))).astype(np.float32))
        x = x.to(dtype).cuda()
        ref = kept(x)
        same_rows(mb.mgrit_q8_pack(x), ref)
        v = oo.q8_unpack(ref.q.cpu().numpy(), ref.scale.cpu().numpy(), cols)
        for out in (F32, BF16):                            # exact in both
            assert np.array_equal(n64(mb.mgrit_q8_unpack(ref, dtype=out)), v)
        big, view = wide(x, 5)                             # odd strides and addresses
        same_rows(mb.mgrit_q8_pack(view), ref)
        big2, view2 = wide(torch.zeros_like(x), 6, 3)
        mb.mgrit_q8_unpack(ref, out=view2)
        assert np.array_equal(n64(view2), v)
        assert torch.isnan(big2[:, :3]).all() and torch.isnan(big2[:, 3 + cols:]).all()


def test_pack_at_the_borders():
    say("pack borders")
    x = torch.zeros(12, 40)
    x[1, 3] = 127.5
    x[2, 3] = float(np.nextafter(np.float32(127.5), np.float32(0)))
    x[3, 3], x[3, 4] = float("inf"), 1.0
    x[4, 5], x[4, 39] = float("nan"), 3.0
    x[5, 0], x[5, 1], x[5, 2] = 2.0 ** -149, -(2.0 ** -126), 2.0 ** -127
    x[6, :4] = torch.tensor([64.0, 0.5, 1.5, -2.5])
    x[7, 0], x[7, 1] = float(np.nextafter(np.float32(127.5 * 2.0 ** 121), np.float32(0))), -1e38
    x[8, 1] = 127.5 * 2.0 ** 121
    x[8, 0] = 2.0 ** -120
    x[0, 39] = torch.finfo(F32).max
    x[9, 0], x[9, 39] = -0.0, float("-inf")
    x[10] = -x[6]
    x[11, 31], x[11, 32] = 5.0, float("nan")               # the neighbouring block is not touched
    # a NaN whose mark lies in its lowest bits only
    x.view(torch.int32)[4, 6] = 0x7f800001
    x = x.cuda()
    ref = kept(x)
    assert list(ref.scale[:, 0].cpu()) == [1, 128, 127, 255, 255, 1, 127, 248, 255, 1, 127, 123] and ref.scale[0, 1] == 255
    same_rows(mb.mgrit_q8_pack(x), ref)
    got, v = n64(mb.mgrit_q8_unpack(ref)), oo.q8_unpack(ref.q.cpu().numpy(), ref.scale.cpu().numpy(), 40)
    assert np.array_equal(got, v, equal_nan=True) and np.isnan(got[3, :32]).all() and not np.isnan(got[11, :32]).any()


def test_rows_behind_the_last_one_stay():
    say("pack into a larger array")
    x = rand(1, 5, 70)
    out = mb.q8_empty((9, 70))
    out.q.fill_(77)
    out.scale.fill_(33)
    mb.mgrit_q8_pack(x, out=out[2:7])
    same_rows(out[2:7], kept(x))
    for part in (out[:2], out[7:]):
        assert (part.q == 77).all() and (part.scale == 33).all()
    y = torch.full((7, 70), 5.0, device="cuda")
    mb.mgrit_q8_unpack(out[2:7], out=y[1:6])
    assert (y[0] == 5).all() and (y[6] == 5).all() and not (y[1:6] == 5).all()


def test_states_keep_their_leading_dimensions():
    say("packed states")
    z = rand(2, 17, 64, 64)
    r = mb.mgrit_q8_pack(z)
    assert r.shape == z.shape and r.rows == 17 * 64
    same_rows(r[3], kept(z[3]))
    assert torch.equal(mb.mgrit_q8_unpack(r[3]), mb.mgrit_q8_unpack(r)[3])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows(dtype):
    say("no rows", dtype)
    x = torch.empty((0, 70), dtype=dtype, device="cuda")
    r = mb.mgrit_q8_pack(x)
    assert mb.mgrit_q8_unpack(r).shape == (0, 70)
    y, mean, rstd = mb.mgrit_layer_norm_forward(x)
    assert y.shape == (0, 70) and mean.shape == (0,)
    junk = [torch.full((70,), 3.0, device="cuda") for _ in range(2)]
    for form in (x, r):
        for t in junk:
            t.fill_(3.0)
        mb.mgrit_layer_norm_backward(x, form, None, mean, rstd, dgamma=junk[0], dbeta=junk[1],
                                     dx_dtype=dtype if form is r else None)
        assert not junk[0].any() and not junk[1].any()
    dW, db = torch.full((6, 70), 3.0, device="cuda"), torch.full((6,), 3.0, device="cuda")
    mb.mgrit_q8_weight_grad(torch.empty((0, 6), dtype=dtype, device="cuda"), r, dW=dW, db=db)
    assert not dW.any() and not db.any()


# ------------------------------------------------------------------ LayerNorm forward
def forward_bounds(x, gamma, beta, y, mean, rstd, out):
    """No sum has more than 48 additions in sequence (32 in a lane, 6 over lanes, up to 16 wavefronts less the first).  The
    mean is corrected by the mean of the differences: 2 u |mean| from its last steps, 48 u of the mean difference.  x - mu
    errs by u of itself and by mu's error, the variance by 50 u, so 1/std by 25 u and 4 u from its own steps."""
    spread = np.abs(x - mean[:, None]).mean(1)
    e_mean = U * (3 * np.abs(mean) + 50 * spread)
    xhat = np.abs(x - mean[:, None]) * rstd[:, None]
    e_hat = 34 * U * xhat + (e_mean * rstd)[:, None]
    e_y = np.abs(gamma) * (e_hat + 2 * U * xhat) + 2 * U * (np.abs(beta) + np.abs(y))
    # a shift of the mean moves the variance in second order only, unless it is of the spread's size
    e_rstd = rstd * (30 * U + (e_mean * rstd) ** 2)
    return e_y * 1.01 + HALF_STEP[out] * (np.abs(y) + e_y), e_mean * 1.01, e_rstd * 1.01


def check_forward(x, gamma, beta, out, eps=1e-5, **kw):
    rows, cols = x.shape
    g = np.ones(cols) if gamma is None else n64(gamma)
    b = np.zeros(cols) if beta is None else n64(beta)
    y, mean, rstd = mb.mgrit_layer_norm_forward(x, gamma, beta, eps=eps, y_dtype=out, **kw)
    ry, rm, rr = oo.norm_forward(n64(x), g, b, eps)
    by, bm, br = forward_bounds(n64(x), g, b, ry, rm, rr, y.dtype)
    close(mean, rm, bm, "mean")
    close(rstd, rr, br, "rstd")
    close(y, ry, by, "y")
    return y, mean, rstd


@pytest.mark.parametrize("x_dtype,y_dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_forward(cols, x_dtype, y_dtype):
    say("norm forward", cols, x_dtype, y_dtype)
    gamma, beta = rand(3, cols, spread=0.3, offset=1.0), rand(4, cols)
    for rows in (1, 5, 67):
        x = rand(rows, rows, cols, spread=2.0, offset=0.7, dtype=x_dtype)
        y, mean, rstd = check_forward(x, gamma, beta, y_dtype)
        # slices of wider rows, odd addresses, outputs beside other data, copies in 8 bits from the same pass
        _, view = wide(x, 9, 3)
        big, out = wide(torch.zeros_like(y), 4, 2)
        keep = [mb.q8_empty((rows, cols)) for _ in range(2)]
        y2, m2, r2 = mb.mgrit_layer_norm_forward(view, gamma, beta, y=out, x_q8=keep[0], y_q8=keep[1])
        assert torch.equal(y2, y) and torch.equal(m2, mean) and torch.equal(r2, rstd)
        assert torch.isnan(big[:, :2]).all() and torch.isnan(big[:, 2 + cols:]).all()
        same_rows(keep[0], kept(x))
        same_rows(keep[1], kept(y))


@pytest.mark.parametrize("cols", [64, 768, 5000])
def test_norm_forward_without_gain_and_in_place(cols):
    say("norm forward plain, in place", cols)
    x = rand(7, 33, cols, offset=-2.0)
    y, _, _ = check_forward(x, None, None, F32)
    check_forward(x, rand(8, cols), None, BF16)
    check_forward(x, None, rand(9, cols), BF16, eps=0.5)
    z = x.clone()
    y2, _, _ = mb.mgrit_layer_norm_forward(z, y=z)
    assert y2 is z and torch.equal(z, y)


@pytest.mark.parametrize("cols", [100, 768, 4096])
def test_norm_forward_far_from_zero_and_flat(cols):
    """A mean of 1000 spreads, rows of one value (variance 0: y = beta), tiny and huge values."""
    say("norm forward offsets", cols)
    gamma, beta = rand(3, cols, offset=1.0), rand(4, cols)
    check_forward(rand(5, 9, cols, offset=1000.0), gamma, beta, F32)
    check_forward(rand(5, 9, cols, spread=1e-12), gamma, beta, F32)
    check_forward(rand(5, 9, cols, spread=1e15), gamma, beta, F32)
    flat = torch.full((4, cols), 3.25, device="cuda")
    y, mean, rstd = mb.mgrit_layer_norm_forward(flat, gamma, beta)
    assert torch.equal(y, beta.expand(4, cols)) and (mean == 3.25).all()


def test_one_bad_row_does_not_touch_the_others():
    say("norm with NaN and infinity")
    for cols in (48, 700, 3000):
        x = rand(5, 21, cols)
        ref = mb.mgrit_layer_norm_forward(x)
        x[4, 7], x[11, 9], x[12, 0] = float("nan"), float("inf"), float("-inf")
        y, mean, rstd = mb.mgrit_layer_norm_forward(x)
        bad = torch.zeros(21, dtype=torch.bool, device="cuda")
        bad[[4, 11, 12]] = True
        assert torch.isnan(y[bad]).all() and torch.isnan(rstd[bad]).all()
        for got, want in zip((y, mean, rstd), ref):
            assert torch.equal(got[~bad], want[~bad])


# ------------------------------------------------------------------ LayerNorm backward
def check_backward(dy, x, gamma, rows_q8=None, eps=1e-5, **kw):
    """x: the input; rows_q8: its 8-bit rows, given to the call in its place."""
    rows, cols = dy.shape
    g = np.ones(cols) if gamma is None else n64(gamma)
    _, mean, rstd = oo.norm_forward(n64(x), 1.0, 0.0, eps)
    mean, rstd = (torch.from_numpy(v.astype(np.float32)).cuda() for v in (mean, rstd))
    xv = n64(x) if rows_q8 is None else oo.q8_unpack(rows_q8.q.cpu().numpy(), rows_q8.scale.cpu().numpy(), cols)
    got = mb.mgrit_layer_norm_backward(dy, x if rows_q8 is None else rows_q8, gamma, mean, rstd, **kw)
    m, r = n64(mean), n64(rstd)
    ref = oo.norm_backward(n64(dy), xv, g, m, r)
    # xhat errs by 3 u of itself, g by u; the two row sums by 50 u of their magnitudes, and what is left by its own steps
    xhat, gd = np.abs((xv - m[:, None]) * r[:, None]), np.abs(n64(dy) * g)
    e_dx = r[:, None] * U * (8 * gd + 56 * gd.mean(1, keepdims=True) + 64 * xhat * (gd * xhat).mean(1, keepdims=True))
    close(got[0], ref[0], e_dx * 1.01 + HALF_STEP[got[0].dtype] * (np.abs(ref[0]) + e_dx), "dx")
    # a column's sum: rows of one slot in sequence (there are at least rows / 768 of them), then slots, blocks and runs
    chain = rows / 768 + 16 + 64 + 16
    a = np.abs(n64(dy))
    close(got[1], ref[1], (chain + 5) * U * (a * xhat).sum(0), "dgamma")
    close(got[2], ref[2], (chain + 1) * U * a.sum(0), "dbeta")
    return got, (mean, rstd)


@pytest.mark.parametrize("x_dtype,y_dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_backward(cols, x_dtype, y_dtype):
    say("norm backward", cols, x_dtype, y_dtype)
    gamma = rand(3, cols, spread=0.3, offset=1.0)
    for rows in (1, 2, 5, 63, 67, 300):
        x, dy = rand(rows, rows, cols, spread=2.0, offset=0.7, dtype=x_dtype), rand(rows + 1, rows, cols, dtype=y_dtype)
        got, (mean, rstd) = check_backward(dy, x, gamma)
        _, xv = wide(x, 9, 3)
        _, dv = wide(dy, 3, 1)
        big, out = wide(torch.zeros_like(x), 4, 2)
        again = mb.mgrit_layer_norm_backward(dv, xv, gamma, mean, rstd, dx=out)
        for p, q in zip(got, again):
            assert torch.equal(p, q)
        assert torch.isnan(big[:, :2]).all() and torch.isnan(big[:, 2 + cols:]).all()


@pytest.mark.parametrize("y_dtype,dx_dtype", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_backward_from_kept_rows(cols, y_dtype, dx_dtype):
    say("norm backward kept", cols, y_dtype, dx_dtype)
    for rows in (1, 5, 63, 67, 300):
        x, dy = rand(rows, rows, cols, spread=2.0, offset=0.7), rand(rows + 1, rows, cols, dtype=y_dtype)
        check_backward(dy, x, rand(3, cols, offset=1.0), kept(x), dx_dtype=dx_dtype)


@pytest.mark.parametrize("rows,cols", [(20000, 64), (9001, 200), (8192, 768), (3001, 2050), (2049, 8192)])
def test_norm_backward_of_many_rows(rows, cols):
    say("norm backward many rows", rows, cols)
    x, dy = rand(1, rows, cols, offset=0.2), rand(2, rows, cols, offset=0.5, dtype=BF16)
    check_backward(dy, x, None)
    check_backward(dy, x, rand(3, cols), kept(x))


@pytest.mark.parametrize("cols", [48, 768, 3000])
@pytest.mark.parametrize("rows", [3, 200])
def test_norm_backward_gives_only_what_is_asked_for(rows, cols):
    """The C entry with each of dx, dgamma and dbeta left out."""
    import ctypes as C
    say("norm backward parts", rows, cols)
    x, dy = rand(1, rows, cols), rand(2, rows, cols)
    _, mean, rstd = mb.mgrit_layer_norm_forward(x)
    want = mb.mgrit_layer_norm_backward(dy, x, None, mean, rstd)
    desc = mb.NormDesc(rows, cols, 0, 0, 1e-5)
    n = mb.mgrit_layer_norm_backward_workspace_bytes(rows, cols)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for mask in range(1, 8):
        out = [torch.full_like(w, 7.0) for w in want]
        at = [o.data_ptr() if mask >> k & 1 else None for k, o in enumerate(out)]
        st = mb.lib().mgrit_layer_norm_backward(C.byref(desc), dy.data_ptr(), cols, x.data_ptr(), cols, None, None, None,
                                                mean.data_ptr(), rstd.data_ptr(), at[0], cols, at[1], at[2],
                                                None if mask == 1 else ws.data_ptr(), 0 if mask == 1 else n,
                                                torch.cuda.current_stream().cuda_stream)
        assert st == 0
        for k, (o, w) in enumerate(zip(out, want)):
            assert torch.equal(o, w) if mask >> k & 1 else (o == 7).all()


def test_norm_backward_against_differences():
    """The gradient of <c, LayerNorm(x)> along a direction against a difference quotient of the forward pass, both from
    the library: fp32 outputs err by about 40 u of sizes near 1, divided by the step 2^-6; the quotient's own error is of
    the step's square, (2^-6)^2 * |third derivative| (about the cube of |d| / std)."""
    say("norm differences")
    rows, cols, h = 40, 96, 2.0 ** -6
    x, d, c = rand(1, rows, cols, spread=2.0), rand(2, rows, cols, spread=0.5), rand(3, rows, cols)
    gamma, beta = rand(4, cols, offset=1.0), rand(5, cols)
    up, _, _ = mb.mgrit_layer_norm_forward(x + h * d, gamma, beta)
    down, _, _ = mb.mgrit_layer_norm_forward(x - h * d, gamma, beta)
    _, mean, rstd = mb.mgrit_layer_norm_forward(x, gamma, beta)
    dx, _, _ = mb.mgrit_layer_norm_backward(c, x, gamma, mean, rstd)
    quotient = ((n64(up) - n64(down)) / (2 * h) * n64(c)).sum(1)
    slope = (n64(dx) * n64(d)).sum(1)
    size = np.sqrt((n64(c) ** 2).sum(1) * (n64(d) ** 2).sum(1))
    assert np.all(np.abs(quotient - slope) <= size * (h * h + 200 * U / h))


def test_norm_backward_passes_on_what_is_not_finite():
    say("norm backward NaN")
    x, dy = rand(1, 130, 96), rand(2, 130, 96)
    _, mean, rstd = mb.mgrit_layer_norm_forward(x)
    ref = mb.mgrit_layer_norm_backward(dy, x, None, mean, rstd)
    dy[77, 5] = float("inf")
    dx, dg, db = mb.mgrit_layer_norm_backward(dy, x, None, mean, rstd)
    good = torch.arange(130, device="cuda") != 77
    assert torch.equal(dx[good], ref[0][good]) and torch.isnan(dx[77]).any()
    assert torch.isinf(db[5]) and not torch.isfinite(dg[5])
    rest = torch.arange(96, device="cuda") != 5
    assert torch.equal(dg[rest], ref[1][rest]) and torch.equal(db[rest], ref[2][rest])
    # a block of kept rows that stands for NaNs
    bad = x.clone()
    bad[3, 40] = float("nan")
    dx, dg, db = mb.mgrit_layer_norm_backward(rand(2, 130, 96), mb.mgrit_q8_pack(bad), None, mean, rstd)
    assert torch.isnan(dx[3]).all() and torch.isnan(dg[32:64]).all() and not torch.isnan(dg[:32]).any()
    assert torch.isfinite(dx[4:]).all() and torch.isfinite(db).all()


# ------------------------------------------------------------------ weight gradients
def check_weight_grad(dy, x8, scale=1.0, **kw):
    rows, m = dy.shape
    xv = oo.q8_unpack(x8.q.cpu().numpy(), x8.scale.cpu().numpy(), x8.cols)
    dW, db = mb.mgrit_q8_weight_grad(dy, x8, scale=scale, **kw)
    ref_w, ref_b = oo.weight_grad(n64(dy), xv, scale)
    size_w, size_b = np.abs(n64(dy)).T @ np.abs(xv) * abs(scale), np.abs(n64(dy)).sum(0) * abs(scale)
    # every product enters its sum exactly (three parts of an fp32 dy one after the other), 2 u per addition at the worst
    adds = rows * (3 if dy.dtype == F32 else 1) + 64
    close(dW, ref_w, 2 * adds * U * size_w, "dW")
    close(db, ref_b, (rows + 64) * U * size_b, "db")
    # and as a whole: the roundings of partial sums that grow like a random walk, sum over k of k u^2, are u * adds / sqrt(2)
    # of one product's size, so sqrt(adds / 2) u of the result's; twice that and a few steps
    if rows > 1:
        rms = np.sqrt((n64(dy) ** 2).T @ (xv ** 2)) * abs(scale)
        e = np.linalg.norm(n64(dW) - ref_w) / max(np.linalg.norm(rms), 1e-300)
        assert e <= U * (2 * np.sqrt(adds) + 8), f"dW as a whole: {e:.3g}"
    return dW, db


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k", [(1, 1), (3, 5), (8, 8), (16, 33), (64, 64), (100, 70), (128, 128), (129, 127), (130, 260),
                                 (256, 256), (257, 31), (50, 700), (384, 320), (1001, 513)])
def test_weight_grad(m, k, dtype):
    say("weight grad", m, k, dtype)
    for rows in (1, 7, 31, 32, 33, 64, 95, 333):
        check_weight_grad(rand(1, rows, m, dtype=dtype), kept(rand(2, rows, k)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,m,k", [(4096, 256, 256), (12608, 384, 96), (5000, 1000, 515), (2111, 2049, 260), (70001, 64, 40)])
def test_weight_grad_of_many_rows(rows, m, k, dtype):
    """Cut into slices of the token sum."""
    say("weight grad many rows", rows, m, k, dtype)
    check_weight_grad(rand(1, rows, m, dtype=dtype), kept(rand(2, rows, k, offset=0.1)), scale=0.125)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,m,k", [(40, 4111, 4300), (65, 4112, 4300), (777, 2601, 2300), (900, 9000, 1100), (1000, 17413, 1000),
                                      (12608, 2051, 1000)])
def test_weight_grad_of_large_weights(rows, m, k, dtype):
    """The large tiles, with ragged edges either way, whole tiles and slices in one launch; the reference is the product of
    the same values in float64 on the device."""
    say("weight grad large", rows, m, k, dtype)
    dy, x8 = rand(1, rows, m, dtype=dtype), mb.mgrit_q8_pack(rand(2, rows, k))
    xv = mb.mgrit_q8_unpack(x8).double()
    dW, db = mb.mgrit_q8_weight_grad(dy, x8, scale=0.5)
    ref_w, size = 0.5 * dy.double().t().contiguous() @ xv, 0.5 * dy.double().abs().t().contiguous() @ xv.abs()
    adds = rows * (3 if dtype == F32 else 1) + 64
    assert bool(((dW.double() - ref_w).abs() <= 2 * adds * U * size).all())
    rms = (dy.double().square().t().contiguous() @ xv.square()).sum().sqrt() * 0.5
    assert float((dW.double() - ref_w).norm()) <= U * (2 * np.sqrt(adds) + 8) * float(rms)
    close(db, 0.5 * n64(dy).sum(0), 0.5 * (rows + 64) * U * np.abs(n64(dy)).sum(0), "db")


@pytest.mark.parametrize("rows,m,k,dtype", [(8200, 4000, 4030, BF16), (8200, 2047, 4033, F32), (8191, 4000, 4030, BF16)])
def test_weight_grad_of_whole_rounds(rows, m, k, dtype):
    """Tiles that fill the chip without slices: db from all columns of tiles, from 8192 tokens on, and from the first one."""
    test_weight_grad_of_large_weights(rows, m, k, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [24, 200, 256])
def test_weight_grad_of_slices_of_wider_rows(m, dtype):
    say("weight grad strides", m, dtype)
    for rows in (33, 128):
        dy, x8 = rand(1, rows, m, dtype=dtype), kept(rand(2, rows, 96))
        want = check_weight_grad(dy, x8)
        for pad, at in ((1, 0), (8, 8), (7, 3)):
            _, view = wide(dy, pad, at)
            got = mb.mgrit_q8_weight_grad(view, x8)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_weight_grad_keeps_every_bit_of_an_fp32_cotangent():
    """One token and x = +-1: dW is dy itself, whatever its exponent."""
    say("weight grad exact")
    rng = np.random.default_rng(3)
    bits = rng.integers(0, 1 << 23, (1, 300)) | (rng.integers(30, 250, (1, 300)) << 23) | (rng.integers(0, 2, (1, 300)) << 31)
    dy = torch.from_numpy(bits.astype(np.uint32).view(np.float32)).cuda()
    x = torch.where(torch.arange(64, device="cuda") % 2 == 0, 1.0, -1.0)[None]
    dW, db = mb.mgrit_q8_weight_grad(dy, mb.mgrit_q8_pack(x))
    assert torch.equal(dW, dy[0][:, None] * x) and torch.equal(db, dy[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weight_grad_passes_on_what_is_not_finite(dtype):
    say("weight grad NaN", dtype)
    dy, x = rand(1, 70, 40, dtype=dtype), rand(2, 70, 64)
    x[x.abs() < 0.05] = 0.25
    want = mb.mgrit_q8_weight_grad(dy, mb.mgrit_q8_pack(x))
    dy2 = dy.clone()
    dy2[5, 3], dy2[6, 4] = float("inf"), float("nan")
    x8 = mb.mgrit_q8_pack(x)
    dW, db = mb.mgrit_q8_weight_grad(dy2, x8)
    nonzero = mb.mgrit_q8_unpack(x8)[5] != 0
    assert torch.isinf(dW[3][nonzero]).all() and torch.isinf(db[3]) and torch.isnan(dW[4]).all() and torch.isnan(db[4])
    rest = [r for r in range(40) if r not in (3, 4)]
    assert torch.equal(dW[rest], want[0][rest]) and torch.equal(db[rest], want[1][rest])
    x[9, 33] = float("nan")
    dW, db = mb.mgrit_q8_weight_grad(dy, mb.mgrit_q8_pack(x))
    assert torch.isnan(dW[:, 32:]).all() and torch.equal(dW[:, :32], want[0][:, :32]) and torch.equal(db, want[1])


def test_weight_grad_without_bias():
    say("weight grad without db")
    dy, x8 = rand(1, 77, 40), kept(rand(2, 77, 50))
    want, _ = mb.mgrit_q8_weight_grad(dy, x8)
    dW = torch.full((40, 50), 9.0, device="cuda")
    n = mb.mgrit_q8_weight_grad_workspace_bytes(77, 40, 50, F32)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    st = mb.lib().mgrit_q8_weight_grad(77, 40, 50, 0, dy.data_ptr(), 40, x8.q.data_ptr(), x8.scale.data_ptr(), 1.0,
                                       dW.data_ptr(), None, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(dW, want)


# ------------------------------------------------------------------ calls as programs make them
def every_operator(x, dy, gamma, beta, out, ws):
    """One pass of each, into given outputs."""
    mb.mgrit_layer_norm_forward(x, gamma, beta, y=out["y"], mean=out["mean"], rstd=out["rstd"], x_q8=out["xq"], y_q8=out["yq"])
    mb.mgrit_layer_norm_backward(dy, out["xq"], gamma, out["mean"], out["rstd"], dx=out["dx"], dgamma=out["dg"],
                                 dbeta=out["db"], workspace=ws)
    mb.mgrit_q8_weight_grad(dy, out["yq"], dW=out["dW"], db=out["dbias"], workspace=ws)
    mb.mgrit_q8_unpack(mb.mgrit_q8_pack(out["dx"], out=out["dq"]), out=out["dv"])


def outputs(rows, cols):
    e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    return dict(y=e(rows, cols).bfloat16(), mean=e(rows), rstd=e(rows), xq=mb.q8_empty((rows, cols)), yq=mb.q8_empty((rows, cols)),
                dx=e(rows, cols), dg=e(cols), db=e(cols), dW=e(cols, cols), dbias=e(cols), dq=mb.q8_empty((rows, cols)), dv=e(rows, cols))


def tensors(out):
    return [t for v in out.values() for t in ((v.q, v.scale) if isinstance(v, mb.Q8Rows) else (v,))]


def scratch(rows, cols):
    n = max(mb.mgrit_layer_norm_backward_workspace_bytes(rows, cols), mb.mgrit_q8_weight_grad_workspace_bytes(rows, cols, cols, F32))
    return torch.empty(n, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("rows,cols", [(40, 96), (3000, 768)])
def test_captured_calls_replay_bit_identically(rows, cols):
    """Two graphs that share one workspace, replayed in turn with eager work between them."""
    say("capture", rows, cols)
    data = [[rand(10 * k + 1, rows, cols), rand(10 * k + 2, rows, cols), rand(10 * k + 3, cols, offset=1.0), rand(10 * k + 4, cols)]
            for k in range(2)]
    ws, outs = scratch(rows, cols), [outputs(rows, cols) for _ in range(2)]
    for d, o in zip(data, outs):
        every_operator(*d, o, ws)
    torch.cuda.synchronize()
    want = [[t.clone() for t in tensors(o)] for o in outs]
    graphs = []
    for d, o in zip(data, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            every_operator(*d, o, ws)
        graphs.append(g)
    for rep in range(3):
        for o in outs:
            for t in tensors(o):
                t.fill_(rep + 1)
        ws.fill_(255)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            for t, r in zip(tensors(o), w):
                assert torch.equal(t, r), f"replay {rep}"


def test_a_stream_of_its_own():
    """stream=: outputs and workspace belong to the call's stream, and results are those of the current one."""
    say("another stream")
    x, dy = rand(1, 3000, 768), rand(2, 3000, 768)
    def all_of(stream):
        y, mean, rstd = mb.mgrit_layer_norm_forward(x, stream=stream)
        r = mb.mgrit_q8_pack(x, stream=stream)
        return [y, mean, rstd, mb.mgrit_q8_unpack(r, stream=stream), *mb.mgrit_layer_norm_backward(dy, r, None, mean, rstd, stream=stream),
                *mb.mgrit_q8_weight_grad(dy, r, stream=stream)]
    want = all_of(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        got = all_of(s)
        junk = [torch.full((3000, 768), 1e9, device="cuda") for _ in range(4)]        # would land in memory freed too early
        torch.cuda.synchronize()
        for p, q in zip(got, want):
            assert torch.equal(p, q)
        del got, junk


def test_binding_refusals_on_the_device():
    say("binding refusals")
    x = rand(1, 8, 64)
    r = mb.mgrit_q8_pack(x)
    y, mean, rstd = mb.mgrit_layer_norm_forward(x)
    for f in (lambda: mb.mgrit_q8_pack(x.half()), lambda: mb.mgrit_q8_pack(x.t()), lambda: mb.mgrit_q8_pack(x[:, ::2]),
              lambda: mb.mgrit_q8_pack(x.expand(2, 8, 64)), lambda: mb.mgrit_q8_pack(x, out=r[:4]),
              lambda: mb.mgrit_q8_unpack(r, dtype=torch.float16), lambda: mb.mgrit_q8_unpack(r, out=x[:4]),
              lambda: mb.mgrit_layer_norm_forward(x, gamma=mean), lambda: mb.mgrit_layer_norm_forward(x, gamma=mean[:1].expand(64)),
              lambda: mb.mgrit_layer_norm_forward(x, y_dtype=torch.float64), lambda: mb.mgrit_layer_norm_forward(x, x_q8=r[:4]),
              lambda: mb.mgrit_layer_norm_forward(x, mean=rstd[:4]),
              lambda: mb.mgrit_layer_norm_backward(y, x[:4], None, mean, rstd), lambda: mb.mgrit_layer_norm_backward(y, x, None, mean[:4], rstd),
              lambda: mb.mgrit_layer_norm_backward(y, x, None, mean, rstd, dx_dtype=BF16),
              lambda: mb.mgrit_layer_norm_backward(y, x, None, mean, rstd, workspace=mean),
              lambda: mb.mgrit_q8_weight_grad(y[:4], r), lambda: mb.mgrit_q8_weight_grad(y, r, dW=y)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(mb.MgritError, match="invalid argument"):
        mb.mgrit_layer_norm_forward(x, eps=0.0)
    with pytest.raises(mb.MgritError, match="invalid argument"):
        mb.mgrit_layer_norm_backward(y, x, None, mean, rstd, dx=y)
    with pytest.raises(mb.MgritError, match="workspace too small"):
        mb.mgrit_q8_weight_grad(rand(1, 4000, 64), mb.mgrit_q8_pack(rand(2, 4000, 64)), workspace=torch.empty(128, dtype=torch.uint8, device="cuda"))
    with pytest.raises(mb.MgritError, match="unsupported"):
        mb.mgrit_layer_norm_forward(torch.zeros(2, 16385, device="cuda"))


def test_calls_are_profiled():
    say("profile classes")
    x, dy = rand(1, 64, 96), rand(2, 64, 96)
    mb.mgrit_profile_enable(16)
    try:
        r = mb.mgrit_q8_pack(x)
        _, mean, rstd = mb.mgrit_layer_norm_forward(x)
        mb.mgrit_layer_norm_backward(dy, x, None, mean, rstd)
        mb.mgrit_q8_weight_grad(dy, r)
        torch.cuda.synchronize()
        got = mb.mgrit_profile_read()
    finally:
        mb.mgrit_profile_enable(0)
    assert {k: v["launches"] for k, v in got.items()} == {"q8": 1, "norm_fwd": 1, "norm_bwd": 1, "q8_weight_grad": 1}
    assert got["q8_weight_grad"]["flops"] == 2 * 64 * 96 * 96 and got["q8"]["bytes"] == 64 * 96 * 4 + 64 * 3 * 33


# ------------------------------------------------------------------ ranges
@pytest.mark.parametrize("cols", [3, 40, 768, 5000])
def test_norm_forward_of_rows_past_the_range(cols):
    """Squares past fp32: an rstd of 0, y = beta; the rows beside it stay as they are."""
    say("norm past the range", cols)
    x = rand(1, 6, cols)
    want = mb.mgrit_layer_norm_forward(x, beta=torch.full((cols,), 0.25, device="cuda"))
    big = x.clone()
    big[2] *= 1e30
    y, mean, rstd = mb.mgrit_layer_norm_forward(big, beta=torch.full((cols,), 0.25, device="cuda"))
    assert rstd[2] == 0 and (y[2] == 0.25).all() and torch.isfinite(mean).all()
    others = [0, 1, 3, 4, 5]
    for got, ref in zip((y, mean, rstd), want):
        assert torch.equal(got[others], ref[others])


@pytest.mark.parametrize("dtype,size", [(F32, 2.0 ** -112), (F32, 2.0 ** -126), (BF16, 2.0 ** -126)])
def test_weight_grad_of_tiny_cotangents(dtype, size):
    """Cotangents whose parts (fp32) or values (bf16) are below the smallest normal number still count.  One token per sum, so
    that a product is the result.  A bf16 number holds bits down to 2^-133: what of an fp32 cotangent lies below is cut off."""
    say("weight grad, tiny cotangents", dtype, size)
    dy = (rand(1, 1, 130).clamp(-3, 3) * size).to(dtype)
    x = torch.where(rand(2, 1, 70) > 0, 64.0, -64.0)
    dW, db = mb.mgrit_q8_weight_grad(dy, mb.mgrit_q8_pack(x))
    ref = np.outer(n64(dy)[0], n64(x)[0])
    # three parts' products, each exact or rounded to fp32's last step, 2^-149, and two additions of u each
    lost = 2.0 ** -133 if dtype == F32 else 0.0
    close(dW, ref, 2 * U * np.abs(ref) + 3 * 2.0 ** -149 + lost * 64, "dW")
    close(db, n64(dy)[0], 2 * U * np.abs(n64(dy)[0]) + 3 * 2.0 ** -149 + lost, "db")


def far_rows(rows, cols, stride, dtype):
    """Rows `stride` elements apart, NaN-free; only they are initialised."""
    return torch.empty((rows - 1) * stride + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (stride, 1))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_offsets_past_32_bits(dtype):
    """Rows that lie further than 2^32 bytes, and elements, from the first one."""
    say("far rows", dtype)
    x, dy, gamma = rand(1, 6, 200, dtype=dtype), rand(2, 6, 200, dtype=dtype), rand(3, 200)
    stride = (1 << 30) + 3
    fx, fdy, fy = (far_rows(6, 200, stride, dtype) for _ in range(3))
    fx.copy_(x)
    fdy.copy_(dy)
    same_rows(mb.mgrit_q8_pack(fx), mb.mgrit_q8_pack(x))
    want = mb.mgrit_layer_norm_forward(x, gamma)
    got = mb.mgrit_layer_norm_forward(fx, gamma, y=fy)
    for p, q in zip(got, want):
        assert torch.equal(p, q)
    mean, rstd = want[1:]
    for p, q in zip(mb.mgrit_layer_norm_backward(fdy, fx, gamma, mean, rstd, dx=fy), mb.mgrit_layer_norm_backward(dy, x, gamma, mean, rstd)):
        assert torch.equal(p, q)
    r = mb.mgrit_q8_pack(x)
    assert torch.equal(mb.mgrit_q8_unpack(r, out=fy), mb.mgrit_q8_unpack(r, dtype=dtype))
    del fx, fdy, fy, got
    tokens = 300                                           # the stride is the most that is allowed
    far, near, x8 = far_rows(tokens, 100, 1 << 24, dtype), rand(4, tokens, 100, dtype=dtype), mb.mgrit_q8_pack(rand(5, tokens, 60))
    far.copy_(near)
    for p, q in zip(mb.mgrit_q8_weight_grad(far, x8), mb.mgrit_q8_weight_grad(near, x8)):
        assert torch.equal(p, q)
    with pytest.raises(mb.MgritError, match="unsupported"):
        mb.mgrit_q8_weight_grad(far_rows(2, 100, (1 << 24) + 1, dtype), mb.mgrit_q8_pack(rand(5, 2, 60)))
    del far
    torch.cuda.empty_cache()


def test_more_blocks_than_one_launch_takes():
    """2^30 rows and a few more, of one element (2 GB, 34 GB kept): the second launch's rows."""
    say("2^30 + 77 rows")
    rows = (1 << 30) + 77
    x = torch.zeros((rows, 1), dtype=BF16, device="cuda")
    at = torch.tensor([0, 1, 12345, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, rows - 1], device="cuda")
    x[at, 0] = torch.arange(1.0, 8.0, device="cuda").to(BF16)
    r = mb.mgrit_q8_pack(x)
    same_rows(mb.Q8Rows(r.q[at], r.scale[at], 1), kept(x[at]))
    assert torch.equal(mb.mgrit_q8_unpack(r, out=torch.ones_like(x)), x)
    del r, x
    torch.cuda.empty_cache()


def test_binding_refuses_rows_of_more_than_32_bits():
    say("a row of 2^31 elements")
    x = torch.empty((1, 1 << 31), dtype=BF16, device="cuda")
    for f in (lambda: mb.mgrit_q8_pack(x), lambda: mb.mgrit_layer_norm_forward(x), lambda: mb.mgrit_q8_weight_grad(x, mb.mgrit_q8_pack(rand(1, 1, 4)))):
        with pytest.raises(ValueError, match="2\\^31 - 1"):
            f()
    del x
    torch.cuda.empty_cache()


def test_calls_of_two_threads():
    """Two host threads, a stream each."""
    say("two threads")
    data = [(rand(10 + i, 900, 200), rand(20 + i, 900, 200)) for i in range(2)]
    def run(x, dy):
        r = mb.q8_empty(x.shape)
        _, mean, rstd = mb.mgrit_layer_norm_forward(x, x_q8=r)
        return [mean, rstd, r.q, *mb.mgrit_layer_norm_backward(dy, r, None, mean, rstd), *mb.mgrit_q8_weight_grad(dy, r)]
    want = [run(*d) for d in data]
    torch.cuda.synchronize()
    bad = []
    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = run(*data[i])
                s.synchronize()
                bad.extend(1 for p, q in zip(got, want[i]) if not torch.equal(p, q))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_binding_names_what_is_of_the_wrong_kind():
    say("wrong kinds")
    x = rand(1, 4, 64)
    x8 = mb.mgrit_q8_pack(x)
    for f in (lambda: mb.mgrit_q8_weight_grad(x, x), lambda: mb.mgrit_q8_pack(x, out=x), lambda: mb.mgrit_layer_norm_forward(x, y_q8=x)):
        with pytest.raises(ValueError, match="expected Q8Rows, got Tensor"):
            f()
    for f in (lambda: mb.mgrit_q8_unpack(x8, out=x8), lambda: mb.mgrit_layer_norm_forward(x, gamma=x8),
              lambda: mb.mgrit_q8_weight_grad(x, x8, dW=x8), lambda: mb.mgrit_layer_norm_backward(x, x, None, 0.0, 1.0)):
        with pytest.raises(ValueError, match="expected a tensor, got"):
            f()


def test_the_most_rows():
    """2^31 - 1 rows of one element: x = 1 has the mean 1, y = beta, and dbeta counts the rows (a slot's part of them is exact,
    and so are the sums of slots: multiples of the slot's size up to the last)."""
    say("2^31 - 1 rows of LayerNorm")
    rows, one = (1 << 31) - 1, torch.ones(1, device="cuda")
    x = torch.ones((rows, 1), dtype=BF16, device="cuda")
    y, mean, rstd = mb.mgrit_layer_norm_forward(x, one, 0.5 * one)
    assert (y == 0.5).all() and (mean == 1).all()
    ref = mb.mgrit_layer_norm_forward(x[:1], one, 0.5 * one)[2]
    assert (rstd == ref).all()
    dx, dgamma, dbeta = mb.mgrit_layer_norm_backward(x, x, one, mean, rstd, dx=y)
    assert dx is y and (dx == 0).all() and dgamma[0] == 0
    assert abs(float(dbeta[0]) - rows) <= rows * 64 * U
    del x, y, mean, rstd, dx
    torch.cuda.empty_cache()


def test_the_most_tokens():
    """2^31 - 256 tokens of one feature (69 GB kept): sums of ones are exact at that number, a multiple of 256 below 2^32."""
    say("2^31 - 256 tokens of a weight gradient")
    tokens = (1 << 31) - 256
    x8 = mb.q8_empty((tokens, 1))
    x8.q.zero_()
    x8.q[:, 0] = 64
    x8.scale.fill_(121)                                    # 64 * 2^-6
    dy = torch.ones((tokens, 1), dtype=BF16, device="cuda")
    dW, db = mb.mgrit_q8_weight_grad(dy, x8)
    assert float(dW[0, 0]) == tokens and float(db[0]) == tokens
    del x8, dy
    torch.cuda.empty_cache()


def test_a_stream_of_another_device_is_refused():
    say("a stream of another device")
    x, other = rand(1, 4, 64), types.SimpleNamespace(device_index=torch.cuda.current_device() + 1, cuda_stream=0)
    x8 = mb.mgrit_q8_pack(x, stream=torch.cuda.current_stream())
    _, mean, rstd = mb.mgrit_layer_norm_forward(x)
    for f in (lambda: mb.mgrit_q8_pack(x, stream=other), lambda: mb.mgrit_q8_unpack(x8, stream=other),
              lambda: mb.mgrit_layer_norm_forward(x, stream=other), lambda: mb.mgrit_layer_norm_backward(x, x, None, mean, rstd, stream=other),
              lambda: mb.mgrit_q8_weight_grad(x, x8, stream=other)):
        with pytest.raises(ValueError, match="current device"):
            f()


@pytest.mark.parametrize("cols", [(1 << 31) - 1, (1 << 31) - 2, (1 << 31) - 31, (1 << 31) - 32, (1 << 31) - 33])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_longest_rows(cols, dtype):
    """A row of nearly 2^31 elements: its last block ends inside the row, at its end or behind it, where columns pass 32 bits.
    What lies behind the row stays as it was.  Steps are 1 (a 127 in every block), so that all values are whole numbers."""
    say("the longest rows", cols, dtype)
    blocks = mb.mgrit_q8_blocks(cols)
    x8 = mb.q8_empty((1, cols))
    torch.randint(-127, 128, x8.q.shape, dtype=torch.int8, device="cuda", out=x8.q)
    x8.q[0, ::32] = 127
    x8.q[0, cols:] = 0
    x8.scale.fill_(127)
    store = torch.full((cols + 64,), 5.0, dtype=dtype, device="cuda")
    x = store[:cols].view(1, cols)
    mb.mgrit_q8_unpack(x8, out=x)
    assert (store[cols:] == 5).all()
    for at in range(0, cols, 1 << 28):
        n = min(1 << 28, cols - at)
        assert torch.equal(store[at:at + n], x8.q[0, at:at + n].to(dtype)), at
    again = mb.q8_empty((1, cols))
    again.q.fill_(99)
    again.scale.fill_(99)
    mb.mgrit_q8_pack(x, out=again)
    assert again.scale.shape == (1, blocks) and (again.scale == 127).all() and torch.equal(again.q, x8.q)
    del x8, x, store, again
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ finite rows past fp32's range
MOST = float(torch.finfo(F32).max)


def far_out(cols, dtype):
    """Finite rows whose sums, differences or squares pass fp32's range, whatever their length, and ordinary ones between them.
    Returns (x, the rows that are far out and flat, far out and not flat)."""
    x = rand(cols, 19, cols, spread=2.0)
    most = MOST if dtype == F32 else float(torch.finfo(BF16).max)
    g = rand(7, cols)
    x[1] = 1e38 + 1e37 * g.clamp(-9, 9)                    # one sign: the sum
    x[3] = -x[1]
    x[4] = 3e38 * g.clamp(-1, 1)                           # both: differences
    x[6] = most
    x[7] = -most
    x[9] = most * torch.where(torch.arange(cols, device="cuda") % 2 == 0, 1.0, -1.0)
    x[10] = 0.0
    x[10, cols // 2] = 2.5e38                              # one large value
    x[12] = 1e30
    x[13] = 1e30 * g
    x[15] = 1e24 * g + 1e25
    x[16, 0] = -most
    steep = [1, 3, 4, 9, 10, 13, 15, 16]
    return x.to(dtype), [6, 7, 12] + (steep if cols == 1 else []), [] if cols == 1 else steep


@pytest.mark.parametrize("x_dtype,y_dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 33, 64, 100, 128, 129, 768, 1000, 2050, 4096, 5000, 8192, 8200, 16383, 16384])
def test_norm_of_finite_rows_past_the_range(cols, x_dtype, y_dtype):
    """Such a row has its mean, an rstd of 0 and y = beta (a flat one: its own rstd); NaNs come from NaNs and infinities only.
    And back: its xhat is 0, so that dx is 0 and dgamma that of the other rows."""
    say("norm of far rows", cols, x_dtype, y_dtype)
    gamma, beta = rand(3, cols, offset=1.0), rand(4, cols)
    x, flat, steep = far_out(cols, x_dtype)
    near = [r for r in range(19) if r not in flat + steep]
    kx, ky = mb.q8_empty(x.shape), mb.q8_empty(x.shape)
    y, mean, rstd = mb.mgrit_layer_norm_forward(x, gamma, beta, y_dtype=y_dtype, x_q8=kx, y_q8=ky)
    same_rows(kx, kept(x))
    same_rows(ky, kept(y))
    xs = n64(x)
    # the mean's bound is that of ordinary rows: its sums are of numbers scaled by a power of two
    ref, spread = xs.mean(1), np.abs(xs - xs.mean(1, keepdims=True)).mean(1)
    close(mean, ref, 1.01 * U * (3 * np.abs(ref) + 50 * spread), "mean")
    assert (rstd[steep] == 0).all()
    assert torch.equal(rstd[flat], mb.mgrit_layer_norm_forward(torch.zeros_like(x), gamma, beta)[2][:len(flat)])
    for r in flat + steep:
        assert torch.equal(y[r], beta.to(y_dtype)), r
    alone = mb.mgrit_layer_norm_forward(x[near].contiguous(), gamma, beta, y_dtype=y_dtype)
    for got, want in zip((y, mean, rstd), alone):
        assert torch.equal(got[near], want)
    if x_dtype == y_dtype:                                 # in place: the row is read again before it is written
        z = x.clone()
        assert torch.equal(mb.mgrit_layer_norm_forward(z, gamma, beta, y=z)[0], y)
    # backward, from x and from its 8-bit rows (not those whose blocks stand for NaNs, nor flat ones, which are flat no more)
    dy = rand(5, 19, cols, dtype=y_dtype)
    m, r = n64(mean), n64(rstd)
    for form, value in ((x, xs), (kx, oo.q8_unpack(kx.q.cpu().numpy(), kx.scale.cpu().numpy(), cols))):
        rows = list(range(19))
        if form is kx:
            rows = [i for i in rows if np.isfinite(value[i]).all() and i not in flat]
            form = mb.Q8Rows(kx.q[rows], kx.scale[rows], cols)
        got = mb.mgrit_layer_norm_backward(dy[rows].contiguous(), form, gamma, mean[rows].contiguous(), rstd[rows].contiguous(),
                                           dx_dtype=x_dtype)
        d, g = n64(dy)[rows], n64(gamma)
        want = oo.norm_backward(d, value[rows], g, m[rows], r[rows])
        xhat, gd = np.abs((value[rows] - m[rows, None]) * r[rows, None]), np.abs(d * g)
        e_dx = r[rows, None] * U * (8 * gd + 56 * gd.mean(1, keepdims=True) + 64 * xhat * (gd * xhat).mean(1, keepdims=True))
        close(got[0], want[0], e_dx * 1.01 + HALF_STEP[x_dtype] * (np.abs(want[0]) + e_dx), "dx")
        close(got[1], want[1], 102 * U * (np.abs(d) * xhat).sum(0), "dgamma")
        close(got[2], want[2], 98 * U * np.abs(d).sum(0), "dbeta")


def test_infinities_and_nans_beside_finite_rows_past_the_range():
    """Rows that share a wavefront: each has what it has alone."""
    say("NaN, infinity and far rows")
    for cols in (3, 40, 100, 768, 5000):
        x = rand(5, 12, cols)
        x[1], x[2, 0], x[3, cols - 1], x[4, 1], x[6] = 3e38, float("nan"), float("inf"), float("-inf"), -3e38
        x[8, 0], x[8, 1] = float("inf"), float("-inf")
        x[9, 0], x[9, 1] = MOST, -MOST
        y, mean, rstd = mb.mgrit_layer_norm_forward(x)
        bad = [2, 3, 4, 8]
        for r in range(12):
            one = mb.mgrit_layer_norm_forward(x[r:r + 1].contiguous())
            if r in bad:
                assert torch.isnan(y[r]).all() and torch.isnan(rstd[r])
            else:
                assert torch.isfinite(y[r]).all() and torch.isfinite(mean[r])
                assert torch.equal(y[r], one[0][0]) and mean[r] == one[1][0] and rstd[r] == one[2][0]
        assert (y[1] == 0).all() and (y[6] == 0).all() and rstd[9] == 0
