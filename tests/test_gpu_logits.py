"""The operators between logits and their gradient on the GPU against their float64 definitions (oracle/logits.py), within
bounds that follow from the arithmetic.

u = 2^-24 is half a step of fp32, relative; sums that are taken in fp32 err by at most (additions in sequence) * u * (sum
of magnitudes); the exponential and logarithm are right to 2 u relative; an output of fewer bits adds half of its step."""
import threading

import numpy as np
import pytest
import torch

from oracle import logits as ol
from paper_2601_09026_amd import binding as mb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16
I32, I64 = torch.int32, torch.int64
WIDTHS = [1, 2, 3, 5, 7, 8, 9, 15, 17, 31, 64, 65, 100, 255, 257, 511, 513, 1000, 1024, 1025, 2047, 2048, 2049, 2056, 4097, 8191, 8193, 10007]
NAN, INF = float("nan"), float("inf")


def say(*a):
    print("[case]", *a, flush=True)


def n64(t):
    return t.detach().double().cpu().numpy()


def logits(seed, rows, cols, dtype=F32, spread=3.0):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((rows, cols)) * spread - 2.0
    z[:, rng.integers(0, cols, max(1, cols // 50))] += 5.0
    return torch.from_numpy(z.astype(np.float32)).to(dtype).cuda()


def floats(seed, *shape, spread=1.0):
    return torch.from_numpy((spread * np.random.default_rng(seed).standard_normal(shape)).astype(np.float32)).cuda()


def ids_of(a, dtype=I64):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def some_tokens(seed, rows, cols):
    t = np.random.default_rng(seed).integers(0, cols, rows)
    t[::7] = -100 if rows > 1 else t[::7]
    return t


def wide(t, pad, at=1):
    """The same rows as a slice of wider ones, starting `at` elements into them; the rest is NaN."""
    big = torch.full((t.shape[0], t.shape[1] + pad), NAN, dtype=t.dtype, device="cuda")
    view = big[:, at:at + t.shape[1]]
    view.copy_(t)
    return big, view


def untouched(big, cols, at):
    return torch.isnan(big[:, :at]).all() and torch.isnan(big[:, at + cols:]).all()


def close(got, ref, bound, what):
    got = n64(got)
    assert got.shape == ref.shape, what
    with np.errstate(invalid="ignore"):
        same = (got == ref) | (np.isnan(got) & np.isnan(ref))
        bad = ~same & ~(np.abs(got - ref) <= bound + 1e-37)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} off, worst "
                           f"{np.nanmax(np.where(same, 0, np.abs(got - ref) / (bound + 1e-37))):.3g} times the bound")


class Bounds:
    """Of a row: y = z / tau, delta = (max - z) / tau >= 0, `drop` and `drop2` the means of delta and delta^2 under p.
    A term exp(-delta) has the rounding of a difference, a product with a rounded constant and the exponential, and is
    rescaled when the running maximum grows: together (8 delta + 2) u and 4 u per rescaling.  A lane has at most 32 additions
    within a chunk and one, with three products, per chunk of 4096 elements and more; lanes, wavefronts and 16 parts follow
    in 26 steps of 6 roundings."""

    def __init__(self, z, tau):
        self.tau = tau
        y = np.asarray(z, np.float64) / tau
        self.lp, self.lse, self.entropy, bad, none = ol.rows(z, tau)
        fine = ~bad & ~none
        with np.errstate(invalid="ignore"):
            self.delta = np.where(fine[:, None], y.max(1, keepdims=True) - y, 0.0)
            self.p = np.where(fine[:, None], np.exp(self.lp), 0.0)
            seen = np.where(self.p > 0, self.delta, 0.0)
            self.drop, self.drop2 = (self.p * seen).sum(1), (self.p * seen ** 2).sum(1)
            self.top = np.where(fine, np.abs(y.max(1)), 0.0)
            lns = np.where(fine, np.abs(self.lse - y.max(1)), 0.0)
            self.adds = 32 + 26 * 6 + 10 * (z.shape[1] // 4096 + 1)
            self.e_s = U * (self.adds + 2 + 8 * self.drop)           # relative, of the sum
            self.e_lns = self.e_s + 3 * U * lns
            self.y = np.abs(np.where(np.isfinite(y), y, 0.0))

    def lse_bound(self):
        return 1.01 * (self.e_lns + U * (self.top + 2 * np.abs(self.lse)))

    def lp_bound(self, at):
        """of ln p at given indices [rows, n]"""
        r = np.arange(len(self.lp))[:, None]
        d = self.delta[r, at]
        return 1.01 * (U * (3 * d + np.abs(self.lp[r, at])) + self.e_lns[:, None])

    def entropy_bound(self):
        t = self.adds * U * self.drop + 8 * U * self.drop2 + 8 * U * self.drop
        return 1.01 * (self.e_lns + t + self.drop * self.e_s + 4 * U * (self.drop + np.abs(self.entropy)))

    def p_rel(self, given):
        """relative, of every p; given: from a log-sum-exp in 32 bits that is exact here, else from the call's own sums"""
        lp = np.where(np.isfinite(self.lp), np.abs(self.lp), 0.0)
        if given:
            return U * (self.y + 5 * lp + 4)
        d = np.where(np.isfinite(self.delta), self.delta, 0.0)
        return U * (3 * d + 5 * lp + 4) + self.e_lns[:, None]

    def gradient(self, ref, dtype, given, slope, mass_p, weights, h=None, entropy=None):
        """ref: the gradient; slope = |cotangent| / tau and mass_p = |its factor of p| per row, weights >= 0 what is added per
        element (before the slope)."""
        rel = self.p_rel(given)
        lp = np.where(np.isfinite(self.lp), np.abs(self.lp), 0.0)
        factor = (slope * mass_p)[:, None] * np.ones_like(self.p)
        e = self.p * factor * (rel + 8 * U)
        e += slope[:, None] * weights * 16 * U
        if h is not None:
            b = np.abs(h)[:, None] / self.tau
            e += self.p * b * ((lp + np.abs(entropy)[:, None]) * (rel + 10 * U) + rel)
            if not given:
                e += self.p * b * self.entropy_bound()[:, None]
        return 1.01 * e + HALF_STEP[dtype] * (np.abs(ref) + 1.01 * e) + 2.0 ** -120 * (factor + 1)


def check_values(z, tokens, k=0, tau=1.0, id_dtype=I64, times=1):
    """mgrit_token_logprobs_forward against the definition; times: with the rows so many times one behind the other."""
    b = Bounds(n64(z), tau)
    many = z if times == 1 else z.repeat(times, 1)
    t = None if tokens is None else ids_of(np.tile(tokens, times), id_dtype)
    r = mb.mgrit_token_logprobs_forward(many, t, top_k=k, temperature=tau)
    def every(x):                                          # (a row's sums are grouped from its first 16-byte address on)
        return np.tile(x, (times,) + (1,) * (x.ndim - 1))
    close(r.lse, every(b.lse), every(b.lse_bound()), "lse")
    close(r.entropy, every(b.entropy), every(b.entropy_bound()), "entropy")
    if tokens is not None:
        ref, _, _ = ol.logprobs(n64(z), tokens, tau)
        at = np.clip(tokens, 0, z.shape[1] - 1)[:, None]
        close(r.logprob, every(ref), every(b.lp_bound(at)[:, 0]), "logprob")
    if k:
        best = ol.largest(n64(z), k)
        assert np.array_equal(r.top_ids.cpu().numpy(), every(best)), "ids"
        close(r.top_logprobs, every(np.take_along_axis(b.lp, best, 1)), every(b.lp_bound(best)), "alternatives")
    return r


# ------------------------------------------------------------------ values
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_values(cols, dtype):
    say("values", cols, dtype)
    for rows, k, tau in ((1, min(cols, 20), 1.0), (5, min(cols, 64), 0.7), (67, min(cols, 3), 1.0), (600, 0, 2.0)):
        if rows * cols > 3e6:
            rows = 520
        z, tokens = logits(cols + rows, rows, cols, dtype), some_tokens(rows, rows, cols)
        r = check_values(z, tokens, k, tau)
        for at in (1, 3):                                  # odd addresses and strides
            _, view = wide(z, 9, at)
            s = check_values(view, tokens, k, tau, I32)
            if k:
                assert torch.equal(s.top_ids.long(), r.top_ids)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [50257, 131072, 262147])
def test_values_of_wide_rows(cols, dtype):
    say("wide rows", cols, dtype)
    for rows, k in ((1, 20), (1, 64), (2, 0), (13, 5)):
        z = logits(rows, rows, cols, dtype)
        check_values(z, some_tokens(rows, rows, cols), k)
        check_values(wide(z, 5, 1)[1], None, k)
        check_values(z, some_tokens(rows, rows, cols), k, times=520 // rows)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [5, 64, 200, 2000, 5000, 9000, 50257])
def test_alternatives_among_equals(cols, dtype):
    """Equal values, sorted rows, rows with little unmasked: the order is by value, then by id."""
    say("equals", cols, dtype)
    rng = np.random.default_rng(cols)
    z = np.zeros((14, cols))
    z[1] = np.arange(cols) // 3
    z[2] = -(np.arange(cols) // 5)
    z[3] = rng.integers(0, 4, cols)
    z[4] = rng.integers(0, 2, cols) * 2.0 - 1
    z[5, ::2] = -0.0
    z[6] = -INF
    z[7] = -INF
    z[7, cols // 2:cols // 2 + 3] = 1.0
    z[8] = np.where(rng.random(cols) < 0.98, -INF, rng.integers(0, 3, cols))
    z[9, cols - 1] = 1.0
    z[10] = -3.389e38
    z[11] = np.where(np.arange(cols) % 2, -3.389e38, 0.0)
    z[12] = np.linspace(-200, 200, cols)
    z[13] = np.linspace(1, -300, cols)
    z = torch.from_numpy(z.astype(np.float32)).to(dtype).cuda()
    tokens = rng.integers(0, cols, 14)
    for k in sorted({min(cols, k) for k in (1, 5, 20, 64)}):
        check_values(z, tokens, k)
        check_values(z, tokens, k, times=40)               # (more rows: other ways to share them out)
        check_values(wide(z, 7, 1)[1], tokens, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [3, 70, 1500, 3000, 50257])
def test_rows_that_are_no_distributions(cols, dtype):
    say("bad rows", cols, dtype)
    z = logits(3, 12, cols, dtype)
    z[1, cols // 2], z[2, 0], z[3, cols - 1], z[4] = NAN, INF, NAN, -INF
    z[5, 0], z[5, 1] = INF, -INF
    z[6] = NAN
    z[7], z[7, 1] = -INF, 2.0
    z[8].view(torch.int32 if dtype is F32 else torch.int16)[1] = -1                    # a NaN with its sign set
    tokens = np.array([0, 1, 1, 1, 1, 1, -5, 1, -1, cols, cols + 7, 2 ** 31 - 1])
    bad = [1, 2, 3, 5, 6, 8]
    k = min(cols, 10)
    for form, t in ((z, tokens), (z.repeat(50, 1), np.tile(tokens, 50))):
        r = mb.mgrit_token_logprobs_forward(form, ids_of(t), top_k=k)
        calm = z.clone()
        calm[bad] = 0.0
        s = mb.mgrit_token_logprobs_forward(calm, top_k=k)
        lp, H, lse = (n64(x)[:12] for x in (r.logprob, r.entropy, r.lse))
        assert np.isnan(lp[[1, 2, 3, 5, 9, 10, 11]]).all() and np.isnan(H[bad]).all() and np.isnan(lse[bad]).all()
        assert (lp[[6, 8]] == 0).all() and lp[4] == -INF and lse[4] == -INF and H[4] == 0 and H[7] == 0 and lp[7] == 0 and lse[7] == 2
        assert (r.top_ids[bad] == -1).all() and torch.isnan(r.top_logprobs[bad]).all()
        assert (r.top_ids[4] == torch.arange(k, device="cuda")).all() and (r.top_logprobs[4] == -INF).all()
        if len(form) == 12:                                # what stands beside them is as without them
            for a, b in ((r.entropy, s.entropy), (r.lse, s.lse), (r.top_ids, s.top_ids), (r.top_logprobs, s.top_logprobs)):
                assert torch.equal(a[[0, 4, 7, 9, 10, 11]], b[[0, 4, 7, 9, 10, 11]])
    h = floats(1, 12)
    for kw in (dict(), dict(g_entropy=h)):
        r, d = mb.mgrit_token_logprobs_step(z, ids_of(tokens), floats(2, 12), **kw)
        e = mb.mgrit_token_logprobs_backward(z, ids_of(tokens), r.lse, floats(2, 12), entropy=r.entropy, **kw)
        for x in (d, e):
            assert torch.isnan(x[[1, 2, 3, 5, 9, 10, 11]]).all() and (x[4] == 0).all() and torch.isfinite(x[[0, 7]]).all()
            assert torch.isnan(x[[6, 8]]).all() if kw else (x[[6, 8]] == 0).all()
    # a student's row without a distribution: infinite loss where the teacher has any, gradient 0
    ids, y = ids_of(np.tile([0, 1], (12, 1))), floats(4, 12, 2)
    loss, lse, d = mb.mgrit_distill_step(z, ids, y)
    e = mb.mgrit_distill_backward(z, ids, y, lse)
    assert torch.isnan(loss[bad]).all() and loss[4] == INF and (loss[7] == INF)
    for x in (d, e):
        assert torch.isnan(x[bad]).all() and (x[4] == 0).all() and torch.isfinite(x[[0, 7, 9]]).all()


@pytest.mark.parametrize("cols", [40, 3000, 50257])
def test_values_of_the_types_range(cols):
    """Masks of the type's lowest value, logits near its ends, quotients that pass the range."""
    say("range", cols)
    for dtype in (F32, BF16):
        most = float(torch.finfo(dtype).max)
        z = logits(5, 8, cols, dtype)
        z[0, ::2] = -most
        z[1], z[2], z[3] = most, -most, -most
        z[3, 1] = most
        z[4] *= 1e30
        z[5] += 1e6
        z[6] = torch.tensor([1e-45, -1e-45], device="cuda").repeat(cols)[:cols].to(dtype)
        z[7, 0] = 3e38
        for tau in (1.0, 0.75, 2.0) if cols > 40 else (1.0, 1e-4, 1e4):
            b = Bounds(n64(z), tau)
            r = mb.mgrit_token_logprobs_forward(z, torch.ones(8, dtype=I64, device="cuda"), temperature=tau)
            with np.errstate(over="ignore"):
                over = np.abs(n64(z).max(1) / tau) > float(torch.finfo(F32).max) * (1 + 2.0 ** -25)
            ok = ~over
            close(r.lse[ok], b.lse[ok], b.lse_bound()[ok], "lse")
            close(r.entropy[ok], b.entropy[ok], b.entropy_bound()[ok], "entropy")
            lp, lse, H = n64(r.logprob), n64(r.lse), n64(r.entropy)
            low = over & (n64(z).max(1) < 0)
            assert (lse[low] == -INF).all() and (H[low] == 0).all() and (lp[low] == -INF).all()
            assert np.isnan(lse[over & ~low]).all() and np.isnan(lp[over & ~low]).all()
            assert np.isfinite(lse[ok]).all() and np.isfinite(H[ok]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [40, 1000, 3000, 9000, 50257, 200001])
def test_sharp_and_shifted_rows(cols, dtype):
    """Rows whose quotients by the temperature are far beyond their differences': values and gradients as of any other."""
    say("sharp rows", cols, dtype)
    rows = 6
    for tau, offset, spread in ((1e-4, 100.0, 2.0), (1.0, 3e5, 200.0), (1e-4, -3e5, 0.05), (0.01, 0.0, 1e5), (1e4, 1e8, 1e5), (1.0, -3e30, 1e24)):
        z = (floats(cols, rows, cols) * spread + offset).to(dtype)
        z[:, 2] = z[:, 1]
        z[1, 3] = z[1].max()
        z[2, ::2] = -INF
        tokens = np.array([0, 3, 1, cols - 1, 2, -1])
        tokens[3] = int(z[3].float().argmax())
        b, g = Bounds(n64(z), tau), floats(1, rows)
        times = 1 if cols > 60000 else 90
        many, t = z.repeat(times, 1), ids_of(np.tile(tokens, times))
        lp, H, lse = ol.logprobs(n64(z), tokens, tau)
        ref = ol.logprobs_gradient(n64(z), tokens, np.where(tokens >= 0, n64(g), 0.0), None, tau)
        weights = np.zeros(z.shape)
        weights[np.arange(rows), np.clip(tokens, 0, None)] = tokens >= 0
        bound = b.gradient(ref, dtype, False, np.abs(n64(g)) * (tokens >= 0) / tau, (tokens >= 0).astype(float), weights)
        lp_bound = b.lp_bound(np.clip(tokens, 0, None)[:, None])[:, 0]
        for zz, tt in ((z, ids_of(tokens)), (many, t)):
            n = len(zz) // rows
            r = mb.mgrit_token_logprobs_forward(zz, tt, top_k=2, temperature=tau)
            s, d = mb.mgrit_token_logprobs_step(zz, tt, g.repeat(n), temperature=tau)
            for x in (r, s):
                for i in (0, n - 1):
                    at = slice(i * rows, (i + 1) * rows)
                    close(x.logprob[at], lp, lp_bound, "logprob")
                    close(x.lse[at], lse, b.lse_bound(), "lse")
                    close(x.entropy[at], H, b.entropy_bound(), "entropy")
            close(d[:rows], ref, bound, "gradient")
            close(d[-rows:], ref, bound, "gradient")
            assert np.array_equal(r.top_ids[:rows].cpu().numpy(), ol.largest(n64(z), 2))
        ids, y = np.stack([tokens.clip(0), np.ones(rows, int)], 1), floats(5, rows, 2) * tau
        q = ol.teacher(ids, n64(y), tau, None, cols)
        rel, e_loss = distill_bounds(b, ids, q, n64(y), tau, False)
        loss_ref, _ = ol.distill(n64(z), ids, n64(y), tau)
        for zz in (z, many):
            n = len(zz) // rows
            args = (zz, ids_of(ids).repeat(n, 1), y.repeat(n, 1))
            for loss in (mb.mgrit_distill_forward(*args, temperature=tau)[0], mb.mgrit_distill_step(*args, temperature=tau)[0]):
                close(loss[:rows], loss_ref, e_loss, "loss")


# ------------------------------------------------------------------ gradients of log probabilities
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", WIDTHS + [50257])
def test_gradients(cols, dtype):
    say("gradients", cols, dtype)
    for rows, tau, with_h in ((1, 1.0, False), (6, 0.7, True), (67, 2.0, False), (130, 1.0, True), (600, 1.0, False)):
        if rows * cols > 3e6:
            continue
        z, tokens = logits(cols + rows, rows, cols, dtype), some_tokens(rows, rows, cols)
        g, h = floats(1, rows), floats(2, rows, spread=0.3) if with_h else None
        t = ids_of(tokens)
        g[torch.from_numpy(tokens < 0).cuda()] = NAN       # (not looked at)
        b = Bounds(n64(z), tau)
        gs = np.where(tokens >= 0, n64(g), 0.0)
        hs = None if h is None else n64(h)
        weights = np.zeros(z.shape)
        weights[np.arange(rows), np.clip(tokens, 0, None)] = tokens >= 0
        slope, mass = np.abs(gs) / tau, (tokens >= 0).astype(float)
        # the backward pass on its own: the statistics are its inputs
        lse32, H32 = torch.from_numpy(b.lse.astype(np.float32)).cuda(), torch.from_numpy(b.entropy.astype(np.float32)).cuda()
        ref = ol.logprobs_gradient(n64(z), tokens, gs, hs, tau, n64(lse32), n64(H32))
        bound = b.gradient(ref, dtype, True, slope, mass, weights, hs, b.entropy)
        kw = dict(g_entropy=h, entropy=H32 if with_h else None, temperature=tau)
        d = mb.mgrit_token_logprobs_backward(z, t, lse32, g, **kw)
        close(d, ref, bound, "backward")
        big, out = wide(torch.zeros_like(z), 6, 3)
        assert torch.equal(mb.mgrit_token_logprobs_backward(z, t, lse32, g, dlogits=out, **kw), d) and untouched(big, cols, 3)
        _, view = wide(z, 9, 1)
        assert torch.equal(mb.mgrit_token_logprobs_backward(view, t.to(I32), lse32, g, **kw), d)
        own = z.clone()
        assert mb.mgrit_token_logprobs_backward(own, t, lse32, g, dlogits=own, **kw) is own and torch.equal(own, d)
        # and in one call with the values
        ref = ol.logprobs_gradient(n64(z), tokens, gs, hs, tau)
        bound = b.gradient(ref, dtype, False, slope, mass, weights, hs, b.entropy)
        r, d = mb.mgrit_token_logprobs_step(z, t, g, g_entropy=h, temperature=tau)
        close(d, ref, bound, "step")
        close(r.lse, b.lse, b.lse_bound(), "step's lse")
        close(r.entropy, b.entropy, b.entropy_bound(), "step's entropy")
        lp, _, _ = ol.logprobs(n64(z), tokens, tau)
        close(r.logprob, lp, b.lp_bound(np.clip(tokens, 0, None)[:, None])[:, 0], "step's logprob")
        big, view = wide(z, 8, 5)
        s, e = mb.mgrit_token_logprobs_step(view, t, g, g_entropy=h, temperature=tau, dlogits=view)
        assert e is view and untouched(big, cols, 5)
        close(e, ref, bound, "step in place")
        close(s.logprob, lp, b.lp_bound(np.clip(tokens, 0, None)[:, None])[:, 0], "logprob in place")


# ------------------------------------------------------------------ distillation
def lists(seed, rows, cols, kept):
    """Ragged lists: full ones, short ones, gaps, none, ids that come twice or more often."""
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, cols, (rows, kept))
    for r in range(rows):
        if r % 5 == 1:
            ids[r, rng.integers(0, kept):] = -1
        elif r % 5 == 2:
            ids[r, rng.random(kept) < 0.4] = -7
        elif r % 5 == 3:
            ids[r] = ids[r, 0]
        elif r % 10 == 4:
            ids[r] = -1
    return ids


def distill_bounds(b, ids, q, y, tau, truncated, lse_t=None):
    """Relative error of q and bound of the loss: the arguments of q's exponentials have 3 roundings, their sum at most 10 in
    sequence, q two more."""
    with np.errstate(invalid="ignore", divide="ignore"):
        live = ids >= 0
        yy = np.where(live, y / tau, -np.inf)
        arg = np.abs(yy - lse_t[:, None]) + np.abs(yy) if truncated else np.abs(yy - yy.max(1, keepdims=True))
        arg = np.where(live & np.isfinite(arg), arg, 0.0)
        rel = U * (4 * arg + 4 * (q * arg).sum(1, keepdims=True) + 24)
        at = np.clip(ids, 0, b.lp.shape[1] - 1)
        r = np.arange(len(ids))[:, None]
        lp = np.where(q > 0, b.lp[r, at], 0.0)
        lnq = np.where(q > 0, np.log(np.where(q > 0, q, 1.0)), 0.0)
        term = q * (np.abs(lnq) + np.abs(lp))
        e = q * (rel + 3 * U * np.abs(lnq) + b.lp_bound(at)) + term * (rel + 20 * U)
    return rel, 1.01 * np.where(q > 0, e, 0.0).sum(1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 2, 5, 10, 64, 100, 1000, 2049, 5000, 10007, 50257])
def test_distillation(cols, dtype):
    say("distillation", cols, dtype)
    for rows, kept, tau, truncated, vt in ((1, 1, 1.0, False, F32), (12, 5, 2.0, False, BF16), (33, 64, 0.7, True, F32), (64, 256, 1.5, False, F32),
                                           (600, 16, 2.0, False, BF16)):
        if rows * cols > 3e6:
            continue
        z, ids = logits(cols + rows, rows, cols, dtype), lists(rows, rows, cols, kept)
        y, g = floats(3, rows, kept, spread=2.0).to(vt), floats(4, rows)
        lse_t = floats(5, rows, spread=0.3) + 4.0 if truncated else None
        t = ids_of(ids, I32 if rows % 2 else I64)
        b = Bounds(n64(z), tau)
        q = ol.teacher(ids, n64(y), tau, None if lse_t is None else n64(lse_t), cols)
        rel, e_loss = distill_bounds(b, ids, q, n64(y), tau, truncated, None if lse_t is None else n64(lse_t))
        ref, _ = ol.distill(n64(z), ids, n64(y), tau, None if lse_t is None else n64(lse_t))
        kw = dict(temperature=tau, teacher_lse=lse_t)
        loss, lse = mb.mgrit_distill_forward(z, t, y, **kw)
        close(loss, ref, e_loss, "loss")
        close(lse, b.lse, b.lse_bound(), "lse")
        none = ~(q != 0).any(1)
        assert (loss[torch.from_numpy(none).cuda()] == 0).all()
        _, view = wide(z, 9, 1)
        close(mb.mgrit_distill_forward(view, t, y, **kw)[0], ref, e_loss, "loss of a slice")
        weights, wrel = np.zeros(z.shape), np.zeros(z.shape)
        for r in range(rows):
            for j in np.flatnonzero(q[r] > 0):
                weights[r, ids[r, j]] += q[r, j]
                wrel[r, ids[r, j]] += q[r, j] * (rel[r, j] + 260 * U)       # (equal ids are added up in sequence)
        slope, mass = np.abs(n64(g)) / tau, q.sum(1)
        e_mass = (q * rel).sum(1) + 12 * U * mass

        def bound(ref, given):
            e = b.gradient(ref, dtype, given, slope, mass, weights)
            return e + 1.02 * slope[:, None] * (b.p * e_mass[:, None] + wrel)
        lse32 = torch.from_numpy(b.lse.astype(np.float32)).cuda()
        tl = None if lse_t is None else n64(lse_t)
        refd = ol.distill_gradient(n64(z), ids, n64(y), n64(g), tau, tl, n64(lse32))
        d = mb.mgrit_distill_backward(z, t, y, lse32, g, **kw)
        close(d, refd, bound(refd, True), "backward")
        assert (d[torch.from_numpy(none).cuda()] == 0).all()
        big, out = wide(torch.zeros_like(z), 6, 3)
        assert torch.equal(mb.mgrit_distill_backward(z, t, y, lse32, g, dlogits=out, **kw), d) and untouched(big, cols, 3)
        own = z.clone()
        assert torch.equal(mb.mgrit_distill_backward(own, t, y, lse32, g, dlogits=own, **kw), d)
        refs = ol.distill_gradient(n64(z), ids, n64(y), n64(g), tau, tl)
        loss, lse, d = mb.mgrit_distill_step(z, t, y, g, **kw)
        close(d, refs, bound(refs, False), "step")
        close(loss, ref, e_loss, "step's loss")
        close(lse, b.lse, b.lse_bound(), "step's lse")
        big, view = wide(z, 8, 5)
        loss, _, e = mb.mgrit_distill_step(view, t, y, g, dlogits=view, **kw)
        assert untouched(big, cols, 5)
        close(e, refs, bound(refs, False), "step in place")
        close(loss, ref, e_loss, "loss in place")


@pytest.mark.parametrize("cols", [12, 3000, 50257])
def test_teachers_that_are_no_distributions(cols):
    say("bad teachers", cols)
    z, y = logits(1, 9, cols), floats(2, 9, 4)
    ids = np.tile([3, 1, 0, 2], (9, 1))
    ids[1, 2], ids[2] = cols, -1
    ids[8, 1] = 2 ** 31 - 1
    y[3, 0], y[4, 1], y[5, 2], y[6] = NAN, INF, -INF, -INF
    y[2, 0] = NAN                                          # (not an id's)
    y[7, 3] = -3.4e38
    t = ids_of(ids)
    ref, _ = ol.distill(n64(z), ids, n64(y))
    q = ol.teacher(ids, n64(y), 1.0, None, cols)
    b = Bounds(n64(z), 1.0)
    nan, zero, fine = [1, 3, 4, 8], [2, 6], [0, 5, 7]
    loss, lse = mb.mgrit_distill_forward(z, t, y)
    loss2, lse2, d2 = mb.mgrit_distill_step(z, t, y)
    d = mb.mgrit_distill_backward(z, t, y, lse)
    close(lse, b.lse, b.lse_bound(), "lse")
    close(lse2, b.lse, b.lse_bound(), "lse")
    for x in (loss, loss2):
        assert torch.isnan(x[nan]).all() and (x[zero] == 0).all()
        _, e = distill_bounds(b, ids, np.nan_to_num(q), np.where(np.isfinite(n64(y)), n64(y), -1e30), 1.0, False)
        close(x[fine], ref[fine], e[fine], "loss")
    for x in (d, d2):
        assert torch.isnan(x[nan]).all() and (x[zero] == 0).all() and torch.isfinite(x[fine]).all()


# ------------------------------------------------------------------ how calls are made
def everything(z, t, g, h, ids, y, stream=None):
    r = mb.mgrit_token_logprobs_forward(z, t, top_k=7, stream=stream)
    d = mb.mgrit_token_logprobs_backward(z, t, r.lse, g, entropy=r.entropy, g_entropy=h, stream=stream)
    s, e = mb.mgrit_token_logprobs_step(z, t, g, g_entropy=h, stream=stream)
    loss, lse = mb.mgrit_distill_forward(z, ids, y, temperature=2.0, stream=stream)
    f = mb.mgrit_distill_backward(z, ids, y, lse, g, temperature=2.0, stream=stream)
    loss2, lse2, k = mb.mgrit_distill_step(z, ids, y, g, temperature=2.0, stream=stream)
    return [*r, d, *s[:3], e, loss, lse, f, loss2, lse2, k]


def operands(rows, cols, dtype=BF16, seed=0):
    return (logits(seed, rows, cols, dtype), ids_of(some_tokens(seed, rows, cols)), floats(seed + 1, rows), floats(seed + 2, rows),
            ids_of(lists(seed, rows, cols, 9)), floats(seed + 3, rows, 9))


SIZES = [(3, 50257), (40, 1000), (600, 5003)]


@pytest.mark.parametrize("rows,cols", SIZES)
def test_results_repeat_bit_for_bit(rows, cols):
    say("repeat", rows, cols)
    for dtype in (F32, BF16):
        ops = operands(rows, cols, dtype)
        one, two = everything(*ops), everything(*ops)
        for a, b in zip(one, two):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows,cols", SIZES)
def test_another_stream(rows, cols):
    say("stream", rows, cols)
    ops = operands(rows, cols)
    ref = everything(*ops)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = everything(*ops, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows,cols", SIZES)
def test_captured_and_replayed(rows, cols):
    say("graph", rows, cols)
    ops = operands(rows, cols)
    everything(*ops)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                     # two graphs of the same operands, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = everything(*ops)
        graphs.append((g, out))
    for seed in (5, 6, 7):
        new = operands(rows, cols, seed=seed)
        for a, b in zip(ops, new):
            a.copy_(b)
        ref = everything(*new)
        for g, out in graphs:
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, ref):
                assert torch.equal(a, b)


def test_calls_from_several_threads():
    say("threads")
    jobs = [operands(rows, cols, seed=i) for i, (rows, cols) in enumerate(SIZES + SIZES)]
    refs = [everything(*j) for j in jobs]
    torch.cuda.synchronize()
    got = [None] * len(jobs)

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            got[i] = everything(*jobs[i])
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    [t.start() for t in threads]
    [t.join() for t in threads]
    for one, ref in zip(got, refs):
        for a, b in zip(one, ref):
            assert torch.equal(a, b)


def test_given_results_and_leading_dimensions():
    say("given results")
    z, t, g, h, ids, y = operands(6, 50257, F32)
    ref = everything(z, t, g, h, ids, y)
    z3, lead = z.view(2, 3, -1), (2, 3)
    new = [torch.full(lead, 7.0, device="cuda") for _ in range(3)]
    top_ids, top = torch.zeros(2, 3, 7, dtype=I64, device="cuda"), torch.zeros(2, 3, 7, device="cuda")
    ws = torch.empty(mb.mgrit_token_logprobs_workspace_bytes(6, 50257, F32, 7), dtype=torch.uint8, device="cuda")
    r = mb.mgrit_token_logprobs_forward(z3, t.view(lead), 7, 1.0, *new, top_ids, top, ws)
    assert r.logprob is new[0] and r.entropy is new[1] and r.lse is new[2] and r.top_ids is top_ids
    for a, b in zip(r, ref):
        assert torch.equal(a.view(-1), b.view(-1))
    s, d = mb.mgrit_token_logprobs_step(z3, t.view(lead), g.view(lead), h.view(lead))
    assert d.shape == z3.shape and s.lse.shape == lead and torch.equal(d.view(6, -1), ref[9])
    loss, lse, k = mb.mgrit_distill_step(z3, ids.view(2, 3, -1), y.view(2, 3, -1), g.view(lead), temperature=2.0)
    assert loss.shape == lead and torch.equal(k.view(6, -1), ref[15])
    # a single row without leading dimensions
    one = mb.mgrit_token_logprobs_forward(z[0], t[0], top_k=7)
    assert one.lse.shape == () and one.top_ids.shape == (7,) and torch.equal(one.top_ids, ref[3][0])
    only = mb.mgrit_token_logprobs_forward(z, top_k=7)
    assert only.logprob is None and torch.equal(only.top_ids, ref[3])


def test_gradients_in_the_logits_own_rows():
    """Logits and gradient as slices of the same wider rows, and one behind the other."""
    say("slices of the same rows")
    for rows, cols, dtype in ((5, 1000, BF16), (3, 3001, F32), (2, 50257, BF16)):
        z, t, g, h, ids, y = operands(rows, cols, dtype)
        big = torch.full((rows, 2 * cols + 8), NAN, dtype=dtype, device="cuda")
        left, right = big[:, :cols], big[:, cols + 8:]
        left.copy_(z)
        lse = mb.mgrit_token_logprobs_forward(left, t).lse
        mb.mgrit_token_logprobs_backward(left, t, lse, g, dlogits=right)
        assert torch.equal(right, mb.mgrit_token_logprobs_backward(left, t, lse, g)) and torch.isnan(big[:, cols:cols + 8]).all()
        mb.mgrit_distill_step(left, ids, y, g, dlogits=right)
        assert torch.equal(right, mb.mgrit_distill_step(left, ids, y, g)[2]) and torch.equal(left, z)
        right.copy_(z)
        mb.mgrit_distill_backward(right, ids, y, lse, g, dlogits=left)
        assert torch.equal(left, mb.mgrit_distill_backward(right, ids, y, lse, g)) and torch.equal(right, z)
        pair = torch.stack([z, z])
        mb.mgrit_token_logprobs_step(pair[0], t, g, dlogits=pair[1])
        assert torch.equal(pair[1], mb.mgrit_token_logprobs_step(pair[0], t, g)[1])
        with pytest.raises(mb.MgritError):
            mb.mgrit_token_logprobs_backward(left, t, lse, g, dlogits=big[:, 1:cols + 1])


def check_steps(rows, some, cols, dtype):
    """Both steps of `rows` rows, `some` different ones over and over, into new memory and in place, against 64 bits."""
    z, tokens = logits(rows, some, cols, dtype), some_tokens(rows + 1, some, cols)
    g, h, ids, y = floats(1, some), floats(2, some, spread=0.3), lists(3, some, cols, 30), floats(4, some, 30)
    g[torch.from_numpy(tokens < 0).cuda()] = 0.0
    times = rows // some
    many, t = z.repeat(times, 1), ids_of(np.tile(tokens, times))
    b, gs, hs = Bounds(n64(z), 1.0), n64(g), n64(h)
    weights = np.zeros(z.shape)
    weights[np.arange(some), np.clip(tokens, 0, None)] = tokens >= 0
    ref = ol.logprobs_gradient(n64(z), tokens, gs, hs)
    bound = b.gradient(ref, dtype, False, np.abs(gs), (tokens >= 0).astype(float), weights, hs, b.entropy)
    lp, _, _ = ol.logprobs(n64(z), tokens)
    q = ol.teacher(ids, n64(y), 1.0, None, cols)
    rel, e_loss = distill_bounds(b, ids, q, n64(y), 1.0, False)
    loss_ref, _ = ol.distill(n64(z), ids, n64(y))
    d_ref = ol.distill_gradient(n64(z), ids, n64(y), gs)
    weights, wrel = np.zeros(z.shape), np.zeros(z.shape)
    for r in range(some):
        for j in np.flatnonzero(q[r] > 0):
            weights[r, ids[r, j]] += q[r, j]
            wrel[r, ids[r, j]] += q[r, j] * (rel[r, j] + 40 * U)
    d_bound = b.gradient(d_ref, dtype, False, np.abs(gs), q.sum(1), weights)
    d_bound = d_bound + 1.02 * np.abs(gs)[:, None] * (b.p * ((q * rel).sum(1) + 12 * U * q.sum(1))[:, None] + wrel)
    for inplace in (False, True):
        own = many.clone()
        r, d = mb.mgrit_token_logprobs_step(own, t, g.repeat(times), h.repeat(times), dlogits=own if inplace else None)
        for i in {0, times - 1}:
            at = slice(i * some, (i + 1) * some)
            close(d[at], ref, bound, "gradient")
            close(r.lse[at], b.lse, b.lse_bound(), "lse")
            close(r.logprob[at], lp, b.lp_bound(np.clip(tokens, 0, None)[:, None])[:, 0], "logprob")
        own = many.clone()
        loss, lse, d = mb.mgrit_distill_step(own, ids_of(ids).repeat(times, 1), y.repeat(times, 1), g.repeat(times), dlogits=own if inplace else None)
        for i in {0, times - 1}:
            at = slice(i * some, (i + 1) * some)
            close(d[at], d_ref, d_bound, "distillation's gradient")
            close(loss[at], loss_ref, e_loss, "loss")
            close(lse[at], b.lse, b.lse_bound(), "lse")


@pytest.mark.parametrize("cols,dtype", [(200001, BF16), (131073, BF16), (65537, F32), (262145, F32)])
def test_steps_of_rows_that_no_block_holds(cols, dtype):
    """The rows' sums in a launch of their own, the gradient in another; in place as well."""
    say("wide steps", cols, dtype)
    for rows in (1, 3, 520):
        if rows > 3 and dtype is F32 and cols > 200000:
            continue
        check_steps(rows, min(rows, 3), cols, dtype)


@pytest.mark.parametrize("rows", [1, 64, 65])
@pytest.mark.parametrize("cols,dtype", [(65536, BF16), (65551, BF16), (131072, BF16), (32768, F32), (32771, F32), (65536, F32)])
def test_steps_of_few_long_rows(cols, dtype, rows):
    """Both sides of where few long rows leave the registers for parts."""
    say("few long rows", rows, cols, dtype)
    check_steps(rows, 5 if rows == 65 else min(rows, 4), cols, dtype)


@pytest.mark.parametrize("cols", [9000, 20000, 30000, 40000, 60000, 100000, 130000])
def test_steps_of_every_block(cols):
    """Rows in the registers of 4, 8 or 16 wavefronts, few and many of them, also where the last vectors are full or nearly so."""
    say("steps by block", cols)
    for dtype in (BF16, F32):
        if dtype is F32 and cols > 65536:
            continue
        for rows, c in ((2, cols), (520, cols), (2, cols // 512 * 512 + 7), (515, cols // 512 * 512)):
            z, tokens = logits(cols, 2, c, dtype), np.array([c - 1, 5])
            g = floats(1, 2)
            times = (rows + 1) // 2
            many, t = z.repeat(times, 1)[:rows], ids_of(np.tile(tokens, times)[:rows])
            b, gs = Bounds(n64(z), 1.0), n64(g)
            weights = np.zeros(z.shape)
            weights[np.arange(2), tokens] = 1.0
            ref = ol.logprobs_gradient(n64(z), tokens, gs)
            bound = b.gradient(ref, dtype, False, np.abs(gs), np.ones(2), weights)
            r, d = mb.mgrit_token_logprobs_step(many, t, g.repeat(times)[:rows])
            lp, _, _ = ol.logprobs(n64(z), tokens)
            for i in (0, rows // 2 - 1):
                close(d[2 * i:2 * i + 2], ref, bound, "gradient")
                close(r.logprob[2 * i:2 * i + 2], lp, b.lp_bound(tokens[:, None])[:, 0], "logprob")
            if c % 8 == 0:                                 # (every row has the same place in its vectors)
                assert torch.equal(d[0::2], d[:1].expand((rows + 1) // 2, -1)) and torch.equal(d[1::2], d[1:2].expand(rows // 2, -1))


def test_no_rows():
    say("no rows")
    for dtype in (F32, BF16):
        z, t = torch.empty((0, 70), dtype=dtype, device="cuda"), torch.empty(0, dtype=I64, device="cuda")
        g, ids, y = torch.empty(0, device="cuda"), torch.empty((0, 3), dtype=I64, device="cuda"), torch.empty((0, 3), device="cuda")
        r = mb.mgrit_token_logprobs_forward(z, t, top_k=4)
        assert r.logprob.shape == (0,) and r.top_ids.shape == (0, 4)
        assert mb.mgrit_token_logprobs_backward(z, t, r.lse, g).shape == (0, 70)
        assert mb.mgrit_token_logprobs_step(z, t, g)[1].shape == (0, 70)
        assert mb.mgrit_distill_step(z, ids, y)[2].shape == (0, 70)


def test_refusals_on_the_device():
    say("refusals")
    z, t, g, h, ids, y = operands(6, 100, F32)
    f, b, d = mb.mgrit_token_logprobs_forward, mb.mgrit_token_logprobs_backward, mb.mgrit_distill_forward
    lse = g
    for call, what in ((lambda: f(z.half(), t), "logits"), (lambda: f(z.t(), t), "logits"), (lambda: f(z, t[:5]), "tokens"),
                       (lambda: f(z, t.float()), "tokens"), (lambda: f(z, t.cpu()), "tokens"), (lambda: f(z, t, 65), "top_k"),
                       (lambda: f(z, t, -1), "top_k"), (lambda: f(z, t, top_ids=t), "top_k"), (lambda: f(z, logprob=g), "tokens"),
                       (lambda: f(z, t, 5, top_ids=torch.zeros(6, 5, dtype=I32, device="cuda")), "top_ids"),
                       (lambda: f(z, t, lse=g.double()), "lse"), (lambda: b(z, t, lse, g[:5]), "g_logprob"),
                       (lambda: b(z, t, lse, g, g_entropy=h), "entropy"), (lambda: b(z, t, lse, g, dlogits=z.bfloat16()), "dlogits"),
                       (lambda: b(z, t, lse, g, dlogits=z[:5]), "dlogits"), (lambda: d(z, ids[:5], y), "teacher_ids"),
                       (lambda: d(z, ids, y[:, :4]), "teacher_logits"), (lambda: d(z, ids, y.half()), "teacher_logits"),
                       (lambda: d(z, ids.t(), y), "teacher_ids"), (lambda: d(z, ids, y, teacher_lse=g[:3]), "teacher_lse"),
                       (lambda: d(z, ids.repeat(1, 40), y.repeat(1, 40)), "256"), (lambda: d(z, ids[0, 0], y), "teacher_ids"),
                       (lambda: f(z, None, 3, logprob=g), "tokens")):
        with pytest.raises(ValueError, match=what):
            call()
    for call in (lambda: f(z, t, temperature=0.0), lambda: f(z, t, temperature=float("nan")), lambda: f(z[:, :3].contiguous(), t, 4),
                 lambda: b(z, t, lse, g, dlogits=z, temperature=-1.0)):
        with pytest.raises(mb.MgritError):
            call()


def test_rows_far_apart():
    """Offsets past 32 bits, in elements and in bytes."""
    say("far apart")
    cols, stride = 3001, 2 ** 31 + 13
    for dtype in (BF16, F32):
        big = torch.empty(2 * stride + cols, dtype=dtype, device="cuda")
        view = big.as_strided((3, cols), (stride, 1))
        z, t, g, h, ids, y = operands(3, cols, dtype)
        view.copy_(z)
        tokens = t.cpu().numpy()
        check_values(view, tokens, 7)
        bd, gs, hs = Bounds(n64(z), 1.0), np.where(tokens >= 0, n64(g), 0.0), n64(h)
        weights = np.zeros(z.shape)
        weights[np.arange(3), np.clip(tokens, 0, None)] = tokens >= 0
        ref = ol.logprobs_gradient(n64(z), tokens, gs, hs)
        bound = bd.gradient(ref, dtype, False, np.abs(gs), (tokens >= 0).astype(float), weights, hs, bd.entropy)
        one = everything(view, t, g, h, ids, y)
        other = everything(z, t, g, h, ids, y)
        assert torch.equal(one[3], other[3])
        close(one[9], ref, bound, "step")
        # (rows of another alignment are added up in another order: the last bits may differ, each is within its bound)
        for i in (12, 15):
            assert float((one[i].float() - other[i].float()).abs().max()) <= 4 * HALF_STEP[dtype] * float(other[i].float().abs().max())
        r, d = mb.mgrit_token_logprobs_step(view, t, g, h, dlogits=view)
        close(view, ref, bound, "step in place")
        del view, big, d
        torch.cuda.empty_cache()


# ------------------------------------------------------------------ as they are used
def test_from_the_last_state_to_its_gradient():
    """A training step's end: LayerNorm of the last state, the head's product, cross entropy and distillation from a teacher's
    alternatives, and back to the state's gradient, against autograd in 64 bits on the same operands."""
    say("end of a training step")
    rows, width, cols, k, tau = 96, 64, 1003, 12, 2.0
    x, W = floats(1, rows, width), floats(2, cols, width, spread=0.3)
    gamma, beta = 1.0 + 0.1 * floats(3, width), 0.1 * floats(4, width)
    tokens = ids_of(some_tokens(5, rows, cols))
    best = mb.mgrit_token_logprobs_forward(logits(6, rows, cols), top_k=k)
    count = float((tokens >= 0).sum())
    a, mean, rstd = mb.mgrit_layer_norm_forward(x, gamma, beta)
    z = a @ W.t()
    r, d1 = mb.mgrit_token_logprobs_step(z, tokens, torch.full((rows,), -1.0 / count, device="cuda"))
    loss, _, d2 = mb.mgrit_distill_step(z, best.top_ids, best.top_logprobs, torch.full((rows,), tau * tau / rows, device="cuda"), temperature=tau)
    dx, dgamma, dbeta = mb.mgrit_layer_norm_backward((d1 + d2) @ W, x, gamma, mean, rstd)
    xd, Wd, gd, bd = (t.double().cpu().requires_grad_() for t in (x, W, gamma, beta))
    ad = torch.nn.functional.layer_norm(xd, (width,), gd, bd)
    zd = ad @ Wd.t()
    live = tokens.cpu() >= 0
    ce = torch.nn.functional.cross_entropy(zd, torch.where(live, tokens.cpu(), -100))
    q = torch.softmax(best.top_logprobs.double().cpu() / tau, 1)
    kl = (q * (q.log() - torch.log_softmax(zd / tau, 1).gather(1, best.top_ids.cpu()))).sum(1)
    (ce + tau * tau * kl.mean()).backward()
    # products of 64 and 1003 terms in fp32: their sums' magnitudes times 1003 u, carried through the LayerNorm's gradient
    assert abs(float(-r.logprob.sum() / count) - float(ce.detach())) < 1e-4 * float(ce.detach())
    assert float((loss.cpu() - kl.detach()).abs().max()) < 1e-4
    for got, ref in ((dx, xd.grad), (dgamma, gd.grad), (dbeta, bd.grad)):
        err = (got.double().cpu() - ref).norm() / ref.norm()
        assert err < 1003 * U, float(err)
