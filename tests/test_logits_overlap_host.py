"""Results of the operators between logits and their gradient that lie on each other, on an argument or on the workspace are refused
before anything is enqueued.  Needs no GPU: the pointers are numbers that are never followed, and every call here is refused (what
may lie side by side, or in an argument's place, runs on the GPU)."""
import pytest

from paper_2601_09026_amd import binding as mb
from test_logits_host import INVALID, P, backward, d_backward, d_forward, d_step, desc, forward, step, teacher

# 4 rows of 40 fp32 logits, 64-bit ids, 5 alternatives, 3 kept: bytes of each array
LOGITS, VALUE, IDS = 640, 16, 32


def with_teacher(call):
    """The call with a teacher's arrays among its keywords."""
    def f(t_ids=20 * P, t_logits=21 * P, t_lse=22 * P, **kw):
        return call(t=teacher(ids=t_ids, logits=t_logits, lse=t_lse), **kw)
    return f


T_READS = dict(t_ids=(20 * P, 96), t_logits=(21 * P, 48), t_lse=(22 * P, 16))
CALLS = {
    "forward": (lambda **kw: forward(**{**dict(k=5, ids=6 * P, top=7 * P), **kw}),
                dict(lp=(3 * P, VALUE), H=(4 * P, VALUE), lse=(5 * P, VALUE), ids=(6 * P, 160), top=(7 * P, 80)), dict(z=(P, LOGITS), tokens=(2 * P, IDS))),
    "backward": (lambda **kw: backward(**{**dict(h=6 * P, H=7 * P, dz=9 * P), **kw}), dict(dz=(9 * P, LOGITS)),
                 dict(tokens=(2 * P, IDS), lse=(3 * P, VALUE), g=(4 * P, VALUE), h=(6 * P, VALUE), H=(7 * P, VALUE))),
    "step": (lambda **kw: step(**{**dict(h=8 * P, dz=9 * P), **kw}), dict(lp=(4 * P, VALUE), H=(5 * P, VALUE), lse=(6 * P, VALUE), dz=(9 * P, LOGITS)),
             dict(z=(P, LOGITS), tokens=(2 * P, IDS), g=(3 * P, VALUE), h=(8 * P, VALUE))),
    "d_forward": (with_teacher(d_forward), dict(loss=(3 * P, VALUE), lse=(4 * P, VALUE)), dict(z=(P, LOGITS), **T_READS)),
    "d_backward": (with_teacher(d_backward), dict(dz=(5 * P, LOGITS)), dict(lse=(3 * P, VALUE), g=(4 * P, VALUE), **T_READS)),
    "d_step": (with_teacher(d_step), dict(loss=(4 * P, VALUE), lse=(5 * P, VALUE), dz=(7 * P, LOGITS)), dict(z=(P, LOGITS), g=(3 * P, VALUE), **T_READS)),
}
PAIRS = [(c, out, other) for c, (_, outs, reads) in CALLS.items() for out in outs for other in {**outs, **reads}
         if other != out and not (out == "dz" and other == "z")]


@pytest.mark.parametrize("call,out,other", PAIRS)
def test_results_on_something_else(call, out, other):
    f, outs, reads = CALLS[call]
    size, (at, other_size) = outs[out][1], {**outs, **reads}[other]
    for by in (8 - size, 8, -8, other_size - 8):
        if by or other_size != size:                       # (a forward pass may put a value where it read one)
            assert f(**{out: at + by}) == INVALID, by
    if out in outs and other in outs:
        assert f(**{out: at}) == INVALID
    if call not in ("forward", "d_forward"):
        assert f(**{out: at}) == INVALID


@pytest.mark.parametrize("by", [4 * 37, 4 * 39, 4 * 97, 4 * 99, 4 * 137, 4 * 197, 4 * 339, -12])
def test_values_across_rows_of_wider_ones(by):
    """4 rows of 40 elements at a distance of 100, 4 values: what reaches into a row's elements."""
    for out in ("lp", "H", "lse"):
        assert forward(z=30 * P, ld=100, **{out: 30 * P + by}) == INVALID
        assert step(z=30 * P, ld=100, **{out: 30 * P + by}) == INVALID and step(dz=30 * P, ldd=100, **{out: 30 * P + by}) == INVALID
    for out in ("loss", "lse"):
        assert d_forward(z=30 * P, ld=100, **{out: 30 * P + by}) == INVALID
        assert d_step(z=30 * P, ld=100, **{out: 30 * P + by}) == INVALID and d_step(dz=30 * P, ldd=100, **{out: 30 * P + by}) == INVALID
    assert backward(dz=30 * P, ldd=100, g=30 * P + by) == INVALID and backward(dz=30 * P, ldd=100, lse=30 * P + by) == INVALID
    assert d_backward(dz=30 * P, ldd=100, g=30 * P + by) == INVALID and d_backward(dz=30 * P, ldd=100, t=teacher(lse=30 * P + by)) == INVALID


def test_workspaces_on_something_else():
    f32 = mb.torch.float32
    cols, W = 200001, 60 * P
    d, wide = desc(rows=4, cols=cols), dict(ld=cols, ws=W)
    far = dict(z=30 * P, tokens=40 * P)                    # (a row takes 0.8 MB)
    need = mb.mgrit_token_logprobs_workspace_bytes(4, cols, f32, 5)
    top = dict(k=5, ids=6 * P, top=7 * P)
    for at in (W, W + need - 8):
        for name in ("tokens", "lp", "H", "lse", "ids", "top", "z"):
            assert forward(d, n=need, **{**wide, **far, **top, name: at}) == INVALID, name
    need = mb.mgrit_token_logprobs_workspace_bytes(4, cols, f32, step=True)
    for at in (W, W + need - 8):
        for name in ("tokens", "lp", "H", "lse", "g", "h", "z", "dz"):
            assert step(d, n=need, ldd=cols, **{**wide, **far, "dz": 50 * P, name: at}) == INVALID, name
    far = dict(z=30 * P)
    need = mb.mgrit_distill_workspace_bytes(4, cols, f32, 3)
    for at in (W, W + need - 8):
        for name in ("t_ids", "t_logits", "t_lse", "loss", "lse", "z"):
            assert with_teacher(d_forward)(d=d, n=need, **{**wide, **far, name: at}) == INVALID, name
    need = mb.mgrit_distill_workspace_bytes(4, cols, f32, 3, step=True)
    for at in (W, W + need - 8):
        for name in ("t_ids", "t_logits", "t_lse", "loss", "lse", "g", "z", "dz"):
            assert with_teacher(d_step)(d=d, n=need, ldd=cols, **{**wide, **far, "dz": 50 * P, name: at}) == INVALID, name
