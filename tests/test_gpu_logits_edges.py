"""The operators between logits and their gradient at the ends of what their arguments may hold: teachers given with a
log-sum-exp, empty batches, statistics whose quotients by the temperature are far beyond their differences."""
import numpy as np
import pytest
import torch

from oracle import logits as ol
from paper_2601_09026_amd import binding as mb
from test_gpu_logits import BF16, F32, HALF_STEP, I32, I64, INF, NAN, U, Bounds, close, distill_bounds, floats, ids_of, lists, logits, n64, say, some_tokens

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ a teacher's log-sum-exp
@pytest.mark.parametrize("values", [F32, BF16])
@pytest.mark.parametrize("cols", [12, 3000, 5000, 50257, 200001])
def test_teachers_with_a_log_sum_exp(cols, values):
    """Values that are no numbers, shares and sums of them beyond fp32's range: NaN for loss and gradient, and nothing of a
    value that belongs to no id."""
    say("teachers with a log-sum-exp", cols, values)
    rows = 14
    z, y, g = logits(1, rows, cols), floats(2, rows, 4).to(values), floats(3, rows)
    lse_t = floats(4, rows, spread=0.2) + 2.0
    ids = np.tile([3, 1, 0, 2], (rows, 1))
    y[1, 0], y[2, 1], y[3, 2], ids[4, 3] = INF, NAN, -INF, cols
    ids[5], y[5] = -1, INF
    ids[6, 1], y[6, 1] = -7, INF
    y[7, 0], lse_t[7] = 200.0, 0.0                         # e^200
    lse_t[8], lse_t[9], lse_t[10] = -INF, INF, NAN
    y[11, 0], y[11, 3], lse_t[11] = 88.5, 88.5, 0.0        # 2.7e38, twice
    y[12] = -INF
    y[13, 0], lse_t[13] = INF, INF
    nan, zero, fine = [1, 2, 4, 7, 8, 10, 11, 13], [5, 9, 12], [0, 3, 6]
    q = ol.teacher(ids, n64(y), 1.0, n64(lse_t), cols)
    assert np.isnan(q).any(1).nonzero()[0].tolist() == nan and (~q.any(1)).nonzero()[0].tolist() == zero
    ref, _ = ol.distill(n64(z), ids, n64(y), 1.0, n64(lse_t))
    d_ref = ol.distill_gradient(n64(z), ids, n64(y), n64(g), 1.0, n64(lse_t))
    b = Bounds(n64(z), 1.0)
    calm = np.where(np.isfinite(n64(y)), n64(y), -1e30), np.where(np.isfinite(n64(lse_t)), n64(lse_t), 0.0)
    rel, e_loss = distill_bounds(b, ids, np.nan_to_num(q), calm[0], 1.0, True, calm[1])
    weights, wrel = np.zeros(z.shape), np.zeros(z.shape)
    for r in fine:
        for j in np.flatnonzero(q[r] > 0):
            weights[r, ids[r, j]] += q[r, j]
            wrel[r, ids[r, j]] += q[r, j] * rel[r, j]
    mass, slope = np.nan_to_num(q).sum(1), np.abs(n64(g))
    for times in (1, 50):
        many = (z.repeat(times, 1), ids_of(ids).repeat(times, 1), y.repeat(times, 1))
        kw = dict(teacher_lse=lse_t.repeat(times))
        loss, lse = mb.mgrit_distill_forward(*many, **kw)
        loss2, _, d2 = mb.mgrit_distill_step(*many, g.repeat(times), **kw)
        d = mb.mgrit_distill_backward(*many, lse, g.repeat(times), **kw)
        for at in {0, (times - 1) * rows}:
            for x in (loss, loss2):
                x = x[at:at + rows]
                assert torch.isnan(x[nan]).all() and (x[zero] == 0).all()
                close(x[fine], ref[fine], e_loss[fine], "loss")
            for x, given in ((d, True), (d2, False)):
                x = x[at:at + rows]
                assert torch.isnan(x[nan]).all() and (x[zero] == 0).all()
                bound = b.gradient(d_ref, F32, given, slope, mass, weights)
                bound = bound + 1.02 * slope[:, None] * (b.p * ((np.nan_to_num(q) * rel).sum(1) + 12 * U * mass)[:, None] + wrel)
                if given:                                  # (the log-sum-exp is the call's own here: half a step of it, and its error)
                    bound = bound + 1.02 * b.p * (slope * mass * (b.lse_bound() + U * np.abs(b.lse)))[:, None]
                close(x[fine], d_ref[fine], bound[fine], "gradient")
