"""The operators between logits and their gradient where a block works on several rows one after the other, where gradients are
written past the caches, and where a row's values go through the workspace with long lists of a teacher.

Some rows are held against the float64 definitions (oracle/logits.py), within the bounds of the arithmetic; all of them against
the same rows in another order or in other calls, bit for bit: a row's results depend on its place modulo 16 bytes alone."""
import numpy as np
import pytest
import torch

from oracle import logits as ol
from paper_2601_09026_amd import binding as mb
from test_gpu_logits import BF16, F32, I32, NAN, U, Bounds, close, distill_bounds, floats, ids_of, lists, n64, say, untouched

pytestmark = pytest.mark.gpu


def many_logits(seed, rows, cols, dtype, at=0, pad=0):
    """A different row each, made on the device; at, pad: a slice of wider rows, the rest of which is NaN."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    z = torch.randn((rows, cols), generator=gen, device="cuda") * 3.0 - 2.0
    z[:, torch.randint(0, cols, (max(1, cols // 50),), generator=gen, device="cuda")] += 5.0
    if not pad:
        return z.to(dtype)
    big = torch.full((rows, cols + pad), NAN, dtype=dtype, device="cuda")
    big[:, at:at + cols] = z.to(dtype)
    return big


def operands(seed, rows, cols, kept):
    """Tokens (one row in seven has none), cotangents, ragged lists with ids that come twice, a teacher's logits and log-sum-exps."""
    rng = np.random.default_rng(seed)
    tokens = rng.integers(0, cols, rows)
    tokens[::7] = -1
    return dict(tokens=tokens, g=floats(seed + 1, rows), h=floats(seed + 2, rows, spread=0.3), ids=lists(seed + 3, rows, cols, kept),
                y=floats(seed + 4, rows, kept, spread=2.0), lse=floats(seed + 5, rows, spread=0.3) + 4.0)


def check_tokens(z, at, o, values, dz, entropies, dtype):
    """Rows `at` of a step over z against the definition."""
    zz, tokens = n64(z[at]), o["tokens"][at]
    b, live = Bounds(zz, 1.0), (o["tokens"][at] >= 0).astype(float)
    g, h = n64(o["g"])[at] * live, n64(o["h"])[at] if entropies else None
    weights = np.zeros(zz.shape)
    weights[np.arange(len(at)), np.clip(tokens, 0, None)] = live
    ref = ol.logprobs_gradient(zz, tokens, g, h)
    close(dz[at], ref, b.gradient(ref, dtype, False, np.abs(g), live, weights, h, b.entropy), "gradient")
    lp, _, _ = ol.logprobs(zz, tokens)
    close(values.logprob[at], lp, b.lp_bound(np.clip(tokens, 0, None)[:, None])[:, 0], "logprob")
    close(values.lse[at], b.lse, b.lse_bound(), "lse")
    close(values.entropy[at], b.entropy, b.entropy_bound(), "entropy")


def check_teacher(z, at, o, loss, lse, dz, truncated, tau, dtype):
    zz, ids, y, g = n64(z[at]), o["ids"][at], n64(o["y"])[at], n64(o["g"])[at]
    t = n64(o["lse"])[at] if truncated else None
    b, q = Bounds(zz, tau), ol.teacher(ids, y, tau, t, zz.shape[1])
    rel, e_loss = distill_bounds(b, ids, q, y, tau, truncated, t)
    close(loss[at], ol.distill(zz, ids, y, tau, t)[0], e_loss, "loss")
    close(lse[at], b.lse, b.lse_bound(), "student's lse")
    if dz is None:
        return
    ref, slope, mass = ol.distill_gradient(zz, ids, y, g, tau, t), np.abs(g) / tau, q.sum(1)
    weights, wrel = np.zeros(zz.shape), np.zeros(zz.shape)
    for r in range(len(at)):
        for j in np.flatnonzero(q[r] > 0):
            weights[r, ids[r, j]] += q[r, j]
            wrel[r, ids[r, j]] += q[r, j] * (rel[r, j] + 260 * U)           # (equal ids are added up in sequence)
    e = b.gradient(ref, dtype, False, slope, mass, weights)
    e = e + 1.02 * slope[:, None] * (b.p * ((q * rel).sum(1) + 12 * U * mass)[:, None] + wrel)
    close(dz[at], ref, e, "distillation's gradient")


def another_order(rows):
    """Groups of 8 rows back to front: each row keeps its place modulo 16 bytes, and has other rows before it in its block."""
    return torch.arange(rows, device="cuda").view(-1, 8).flip(0).reshape(-1)


# rows and columns: as many rows as blocks run at once, twice and a bit more, for each form of rows in registers
WALKS = [(14000, 130, BF16), (14000, 61, F32), (11000, 1500, BF16), (11000, 1001, F32), (11000, 2501, BF16), (9000, 2048, F32),
         (2800, 5000, BF16), (2800, 4001, F32), (2400, 12001, BF16), (2400, 6000, F32), (2200, 30000, BF16), (2200, 16001, F32),
         (1744, 50257, BF16), (1744, 25003, F32), (520, 60001, BF16), (520, 30003, F32), (520, 100000, BF16), (520, 50003, F32),
         (520, 131071, BF16), (520, 65536, F32)]


@pytest.mark.parametrize("rows,cols,dtype", WALKS)
def test_steps_of_many_rows(rows, cols, dtype):
    say("walk", rows, cols, dtype)
    rows, kept = rows // 8 * 8, min(cols, 70)
    z, o = many_logits(rows, rows, cols, dtype), operands(cols, rows, cols, kept)
    t, ids, order = ids_of(o["tokens"]), ids_of(o["ids"], I32), another_order(rows)
    at = np.unique(np.concatenate([[0, 1, 255, 256, 511, 513, rows - 1], np.random.default_rng(rows).integers(0, rows, 7)]))
    for entropies in (False, True):
        h = o["h"] if entropies else None
        r, d = mb.mgrit_token_logprobs_step(z, t, o["g"], g_entropy=h)
        check_tokens(z, at, o, r, d, entropies, dtype)
        s, e = mb.mgrit_token_logprobs_step(z[order], t[order], o["g"][order], g_entropy=None if h is None else h[order])
        assert torch.equal(e, d[order])
        for x, y in zip(s[:3], r[:3]):
            assert torch.equal(x, y[order])
        own = z.clone()
        mb.mgrit_token_logprobs_step(own, t, o["g"], g_entropy=h, dlogits=own)
        assert torch.equal(own, d)
        del d, e, own
    for truncated, tau in ((False, 2.0), (True, 1.0)):
        kw = dict(temperature=tau, teacher_lse=o["lse"] if truncated else None)
        loss, lse, d = mb.mgrit_distill_step(z, ids, o["y"], o["g"], **kw)
        check_teacher(z, at, o, loss, lse, d, truncated, tau, dtype)
        kw2 = dict(kw, teacher_lse=o["lse"][order] if truncated else None)
        loss2, lse2, e = mb.mgrit_distill_step(z[order], ids[order], o["y"][order], o["g"][order], **kw2)
        assert torch.equal(e, d[order]) and torch.equal(loss2, loss[order]) and torch.equal(lse2, lse[order])
        own = z.clone()
        mb.mgrit_distill_step(own, ids, o["y"], o["g"], dlogits=own, **kw)
        assert torch.equal(own, d)
        del d, e, own
    # odd strides and addresses, in place
    for name in ("tokens", "teacher"):
        big = many_logits(rows, rows, cols, dtype, 3, 8)
        view = big[:, 3:3 + cols]
        if name == "tokens":
            r, d = mb.mgrit_token_logprobs_step(view, t, o["g"], g_entropy=o["h"], dlogits=view)
            check_tokens(z, at, o, r, d, True, dtype)
        else:
            loss, lse, d = mb.mgrit_distill_step(view, ids, o["y"], o["g"], temperature=2.0, dlogits=view)
            check_teacher(z, at, o, loss, lse, d, False, 2.0, dtype)
        assert d is view and untouched(big, cols, 3)


@pytest.mark.parametrize("rows,cols,dtype", [w for w in WALKS if w[0] >= 9000])
def test_values_of_many_short_rows(rows, cols, dtype):
    say("walk of values", rows, cols, dtype)
    rows, kept = rows // 8 * 8, min(cols, 70)
    z, o = many_logits(rows, rows, cols, dtype), operands(cols, rows, cols, kept)
    t, ids, order = ids_of(o["tokens"]), ids_of(o["ids"]), another_order(rows)
    at = np.unique(np.concatenate([[0, 1, rows - 1], np.random.default_rng(rows).integers(0, rows, 13)]))
    zz = n64(z[at])
    b, best = Bounds(zz, 1.0), ol.largest(zz, 9)
    lp, _, _ = ol.logprobs(zz, o["tokens"][at])
    for k in (0, 9):
        r = mb.mgrit_token_logprobs_forward(z, t, top_k=k)
        close(r.lse[at], b.lse, b.lse_bound(), "lse")
        close(r.entropy[at], b.entropy, b.entropy_bound(), "entropy")
        close(r.logprob[at], lp, b.lp_bound(np.clip(o["tokens"][at], 0, None)[:, None])[:, 0], "logprob")
        if k:
            assert np.array_equal(r.top_ids[at].cpu().numpy(), best)
            close(r.top_logprobs[at], np.take_along_axis(b.lp, best, 1), b.lp_bound(best), "alternatives")
        s = mb.mgrit_token_logprobs_forward(z[order], t[order], top_k=k)
        for x, y in zip(s[:5 if k else 3], r):
            assert torch.equal(x, y[order])
    for truncated in (False, True):
        kw = dict(temperature=1.0, teacher_lse=o["lse"] if truncated else None)
        loss, lse = mb.mgrit_distill_forward(z, ids, o["y"], **kw)
        check_teacher(z, at, o, loss, lse, None, truncated, 1.0, dtype)
        kw2 = dict(kw, teacher_lse=o["lse"][order] if truncated else None)
        loss2, lse2 = mb.mgrit_distill_forward(z[order], ids[order], o["y"][order], **kw2)
        assert torch.equal(loss2, loss[order]) and torch.equal(lse2, lse[order])


@pytest.mark.parametrize("rows,cols,dtype", [(2800, 50304, BF16), (2800, 50257, BF16), (1440, 50003, F32), (1072, 131077, BF16)])
def test_gradients_past_the_caches(rows, cols, dtype):
    """Gradients of more than 256 MiB, against the definition and against calls of half the rows, which are written the ordinary way
    (1072 x 131077: through the workspace)."""
    say("past the caches", rows, cols, dtype)
    size, half = 2 if dtype is BF16 else 4, rows // 2
    assert rows * cols * size > 256 << 20 > half * cols * size and half % 8 == 0 and half > 512
    z, o = many_logits(rows, rows, cols, dtype), operands(cols, rows, cols, 40)
    t, ids = ids_of(o["tokens"]), ids_of(o["ids"])
    at = np.unique(np.concatenate([[0, 1, half - 1, half, rows - 1], np.random.default_rng(rows).integers(0, rows, 5)]))
    halves = (slice(0, half), slice(half, rows))

    def both(call, *per_row):
        """The call's results, and those of the halves and in place, which are the same."""
        whole = call(z, None, *per_row)
        for x in halves:
            part = call(z[x], None, *(None if p is None else p[x] for p in per_row))
            for a, b in zip(whole, part):
                assert torch.equal(a[x], b)
            del part
        own = z.clone()
        for a, b in zip(whole, call(own, own, *per_row)):
            assert torch.equal(a, b)
        return whole

    for h in (None, o["h"]):
        def step(z, out, t, g, h):
            r, d = mb.mgrit_token_logprobs_step(z, t, g, g_entropy=h, dlogits=out)
            return d, r.logprob, r.entropy, r.lse
        d, *r = both(step, t, o["g"], h)
        check_tokens(z, at, o, mb.TokenLogprobs(*r), d, h is not None, dtype)
        entropy, lse = r[1], r[2]

        def backward(z, out, t, lse, g, entropy, h):
            return mb.mgrit_token_logprobs_backward(z, t, lse, g, entropy=entropy, g_entropy=h, dlogits=out),
        (e,) = both(backward, t, lse, o["g"], entropy, h)
        zz, tokens = n64(z[at]), o["tokens"][at]
        b, live = Bounds(zz, 1.0), (tokens >= 0).astype(float)
        g, hs = n64(o["g"])[at] * live, None if h is None else n64(h)[at]
        weights = np.zeros(zz.shape)
        weights[np.arange(len(at)), np.clip(tokens, 0, None)] = live
        ref = ol.logprobs_gradient(zz, tokens, g, hs, 1.0, n64(lse)[at], n64(entropy)[at])
        close(e[at], ref, b.gradient(ref, dtype, True, np.abs(g), live, weights, hs, b.entropy), "backward")
        del d, e

    def distill(z, out, ids, y, g):
        loss, lse, d = mb.mgrit_distill_step(z, ids, y, g, temperature=2.0, dlogits=out)
        return d, loss, lse
    d, loss, lse = both(distill, ids, o["y"], o["g"])
    check_teacher(z, at, o, loss, lse, d, False, 2.0, dtype)

    def back(z, out, ids, y, lse, g):
        return mb.mgrit_distill_backward(z, ids, y, lse, g, temperature=2.0, dlogits=out),
    del d
    both(back, ids, o["y"], lse, o["g"])


@pytest.mark.parametrize("rows,cols,dtype", [(1, 131072, BF16), (3, 200001, BF16), (64, 70001, F32), (520, 131077, BF16), (2, 600001, F32)])
def test_long_lists_through_the_workspace(rows, cols, dtype):
    """More ids of a teacher than a wavefront has lanes, with and without its log-sum-exp, where a step's values lie in the workspace."""
    say("long lists", rows, cols, dtype)
    assert mb.mgrit_distill_workspace_bytes(rows, cols, dtype, 256, step=True) > 0
    z = many_logits(rows, rows, cols, dtype)
    at = np.unique([0, 1 % rows, 2 % rows, rows // 2, rows - 1])
    for kept in (65, 200, 256):
        o = operands(cols + kept, rows, cols, kept)
        o["ids"][0] = np.random.default_rng(kept).integers(0, cols, kept)
        o["ids"][0, -1] = o["ids"][0, 3]
        ids = ids_of(o["ids"])
        for truncated in (False, True):
            kw = dict(teacher_lse=o["lse"] if truncated else None, temperature=1.5)
            loss, lse, d = mb.mgrit_distill_step(z, ids, o["y"], o["g"], **kw)
            check_teacher(z, at, o, loss, lse, d, truncated, 1.5, dtype)
            loss, lse = mb.mgrit_distill_forward(z, ids, o["y"], **kw)
            check_teacher(z, at, o, loss, lse, None, truncated, 1.5, dtype)
            own = z.clone()
            mb.mgrit_distill_step(own, ids, o["y"], o["g"], dlogits=own, **kw)
            assert torch.equal(own, d)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [40, 1000, 3000, 5000, 9000, 30000, 50257, 60001, 131075])
def test_steps_of_sharp_and_shifted_rows(cols, dtype):
    """Gradients, with entropies and of distillation, of rows whose quotients by the temperature are far beyond their differences,
    in every form of rows in registers and through the workspace."""
    say("steps of sharp rows", cols, dtype)
    rows = 6
    times = (1, 200) if cols < 60000 else (1, 90)
    for tau, offset, spread in ((1e-4, 100.0, 2.0), (1.0, 3e5, 200.0), (0.7, 3e5, 20.0), (0.01, -3e3, 0.5), (1e4, 1e8, 1e5), (3.0, -3e30, 1e24)):
        tau = float(np.float32(tau))
        z = (floats(cols, rows, cols) * spread + offset).to(dtype)
        z[:, 2] = z[:, 1]
        z[1, 3] = z[1].max()
        z[2, ::2] = -float("inf")
        tokens = np.array([0, 3, 1, cols - 1, 2, -1])
        tokens[3] = int(z[3].float().argmax())
        g, h, zz, b = floats(1, rows), floats(2, rows, spread=0.3), n64(z), Bounds(n64(z), tau)
        live = (tokens >= 0).astype(float)
        gs, hs, slope = n64(g) * live, n64(h), np.abs(n64(g)) / tau
        weights = np.zeros(z.shape)
        weights[np.arange(rows), np.clip(tokens, 0, None)] = live
        ref = ol.logprobs_gradient(zz, tokens, gs, hs, tau)
        bound = b.gradient(ref, dtype, False, slope * live, live, weights, hs, b.entropy)
        # (a p below 2^-126 counts as 0; its factor is at most |h| / tau (88 + H))
        bound = bound + 2.0 ** -126 * (np.abs(hs) / tau * (88 + b.entropy))[:, None]
        ids, y = np.stack([tokens.clip(0), np.ones(rows, int), np.full(rows, cols // 2)], 1), floats(5, rows, 3) * tau
        q = ol.teacher(ids, n64(y), tau, None, cols)
        rel, e_loss = distill_bounds(b, ids, q, n64(y), tau, False)
        d_ref, loss_ref = ol.distill_gradient(zz, ids, n64(y), n64(g), tau), ol.distill(zz, ids, n64(y), tau)[0]
        weights, wrel = np.zeros(z.shape), np.zeros(z.shape)
        for r in range(rows):
            for j in range(3):
                weights[r, ids[r, j]] += q[r, j]
                wrel[r, ids[r, j]] += q[r, j] * (rel[r, j] + 3 * U)
        d_bound = b.gradient(d_ref, dtype, False, slope, q.sum(1), weights)
        d_bound = d_bound + 1.02 * slope[:, None] * (b.p * ((q * rel).sum(1) + 12 * U)[:, None] + wrel)
        for n in times:
            many, gn = z.repeat(n, 1), g.repeat(n)
            _, d = mb.mgrit_token_logprobs_step(many, ids_of(np.tile(tokens, n)), gn, g_entropy=h.repeat(n), temperature=tau)
            loss, _, e = mb.mgrit_distill_step(many, ids_of(ids).repeat(n, 1), y.repeat(n, 1), gn, temperature=tau)
            for at in {0, (n - 1) * rows}:
                close(d[at:at + rows], ref, bound, "gradient")
                close(e[at:at + rows], d_ref, d_bound, "distillation's gradient")
                close(loss[at:at + rows], loss_ref, e_loss, "loss")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_longest_rows(dtype):
    """2^24 logits a row, whole and in slices at odd addresses: values, alternatives and both steps."""
    cols, rows, kept = 2 ** 24, 2, 100
    say("longest rows", dtype)
    z, o = many_logits(1, rows, cols, dtype), operands(2, rows, cols, kept)
    o["tokens"][:] = cols - 1, 5
    o["ids"][1] = np.random.default_rng(3).integers(0, cols, kept)
    o["ids"][:, 0] = cols - 1
    t, ids, at = ids_of(o["tokens"]), ids_of(o["ids"]), np.arange(rows)
    b, best = Bounds(n64(z), 1.0), ol.largest(n64(z), 64)
    r = mb.mgrit_token_logprobs_forward(z, t, 64)
    close(r.lse, b.lse, b.lse_bound(), "lse")
    close(r.entropy, b.entropy, b.entropy_bound(), "entropy")
    assert np.array_equal(r.top_ids.cpu().numpy(), best)
    close(r.top_logprobs, np.take_along_axis(b.lp, best, 1), b.lp_bound(best), "alternatives")
    s, d = mb.mgrit_token_logprobs_step(z, t, o["g"], o["h"])
    check_tokens(z, at, o, s, d, True, dtype)
    loss, lse, d = mb.mgrit_distill_step(z, ids, o["y"], o["g"])
    check_teacher(z, at, o, loss, lse, d, False, 1.0, dtype)
    big = many_logits(1, rows, cols, dtype, 3, 8)
    view = big[:, 3:3 + cols]
    loss, lse, d = mb.mgrit_distill_step(view, ids, o["y"], o["g"], dlogits=view)
    check_teacher(z, at, o, loss, lse, d, False, 1.0, dtype)
    assert untouched(big, cols, 3)


@pytest.mark.parametrize("rows,cols,dtype", [(2 ** 24 + 40, 3, F32), (2 ** 24 + 40, 5, BF16), (2 ** 22 + 8, 4104, BF16)])
def test_more_rows_than_blocks_along_x(rows, cols, dtype):
    """8 rows over and over, more often than a launch has blocks in one direction: all have the results of the first 8."""
    say("many rows", rows, cols, dtype)
    z, o = many_logits(1, 8, cols, dtype), operands(2, 8, cols, 3)
    times = rows // 8
    assert rows % 8 == 0
    t, ids = ids_of(o["tokens"], I32), ids_of(o["ids"], I32)
    many = [x.repeat(times, *[1] * (x.dim() - 1)) for x in (z, t, o["g"], o["h"], ids, o["y"])]

    def same(x, first):
        """In pieces: the comparison's own memory stays small."""
        for part in x.view(times, *first.shape).split(2 ** 16):
            assert torch.equal(part, first.expand_as(part))
    r = mb.mgrit_token_logprobs_forward(many[0], many[1], 3)
    for x in r:
        same(x, x[:8].clone())
    at = np.arange(8)
    b, best = Bounds(n64(z), 1.0), ol.largest(n64(z), 3)
    close(r.lse[:8], b.lse, b.lse_bound(), "lse")
    assert np.array_equal(r.top_ids[:8].cpu().numpy(), best)
    loss, lse = mb.mgrit_distill_forward(many[0], many[4], many[5])
    check_teacher(z, at, o, loss[:8], lse[:8], None, False, 1.0, dtype)
    same(loss, loss[:8].clone())
    H, lse, entropy = many[3], r.lse, r.entropy
    zz, g, h = n64(z), n64(o["g"]) * (o["tokens"] >= 0), n64(o["h"])
    weights, live = np.zeros(zz.shape), (o["tokens"] >= 0).astype(float)
    weights[at, np.clip(o["tokens"], 0, None)] = live
    ref = ol.logprobs_gradient(zz, o["tokens"], g, h, 1.0, n64(lse[:8]), n64(entropy[:8]))
    # (in place: the gradient replaces the logits, which come back behind it)
    d = mb.mgrit_token_logprobs_backward(many[0], many[1], lse, many[2], entropy=entropy, g_entropy=H, dlogits=many[0])
    close(d[:8], ref, b.gradient(ref, dtype, True, np.abs(g), live, weights, h, b.entropy), "backward")
    same(d, d[:8].clone())
    many[0].view(times, 8, cols).copy_(z.expand(times, 8, cols))
    s, d = mb.mgrit_token_logprobs_step(many[0], many[1], many[2], H, dlogits=many[0])
    check_tokens(z, at, o, s, d, True, dtype)
    same(d, d[:8].clone())
    many[0].view(times, 8, cols).copy_(z.expand(times, 8, cols))
    d = mb.mgrit_distill_backward(many[0], many[4], many[5], lse, many[2], dlogits=many[0])
    same(d, d[:8].clone())
    many[0].view(times, 8, cols).copy_(z.expand(times, 8, cols))
    loss, lse, d = mb.mgrit_distill_step(many[0], many[4], many[5], many[2], dlogits=many[0])
    check_teacher(z, at, o, loss[:8], lse[:8], d[:8], False, 1.0, dtype)
    same(d, d[:8].clone())
    del many, d
    torch.cuda.empty_cache()
