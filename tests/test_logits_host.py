"""What the operators between logits and their gradient refuse, before anything is enqueued.  Needs no GPU: the pointers are
numbers that are never followed."""
import ctypes as C

import pytest
import torch

from paper_2601_09026_amd import binding as mb

INVALID, UNSUPPORTED, SMALL, OK = mb.MGRIT_INVALID_ARG, mb.MGRIT_UNSUPPORTED, mb.MGRIT_WORKSPACE_TOO_SMALL, mb.MGRIT_OK
P = 1 << 20                                               # an aligned address
NAN, INF = float("nan"), float("inf")


def desc(rows=4, cols=40, dtype=0, ids=1, tau=1.0):
    return mb.LogitsDesc(rows, cols, dtype, ids, tau)


def teacher(kept=3, dtype=0, ids=20 * P, logits=21 * P, lse=None):
    return mb.Teacher(kept, dtype, ids, logits, lse)


BAD_DESCS = [(dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(dtype=2), INVALID), (dict(ids=2), INVALID), (dict(ids=-1), INVALID),
             (dict(tau=0.0), INVALID), (dict(tau=-1.0), INVALID), (dict(tau=NAN), INVALID), (dict(tau=INF), INVALID),
             (dict(tau=0.9e-4), INVALID), (dict(tau=1.1e4), INVALID), (dict(cols=(1 << 24) + 1), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED)]
WIDE = 1 << 25


def forward(d=None, z=P, ld=40, tokens=2 * P, lp=3 * P, H=4 * P, lse=5 * P, k=0, ids=None, top=None, ws=None, n=0):
    return mb.lib().mgrit_token_logprobs_forward(desc() if d is None else d, z, ld, tokens, lp, H, lse, k, ids, top, ws, n, None)


def backward(d=None, z=P, ld=40, tokens=2 * P, lse=3 * P, g=4 * P, H=None, h=None, dz=5 * P, ldd=40):
    return mb.lib().mgrit_token_logprobs_backward(desc() if d is None else d, z, ld, tokens, lse, g, H, h, dz, ldd, None)


def step(d=None, z=P, ld=40, tokens=2 * P, g=3 * P, h=None, lp=4 * P, H=5 * P, lse=6 * P, dz=7 * P, ldd=40, ws=None, n=0):
    return mb.lib().mgrit_token_logprobs_step(desc() if d is None else d, z, ld, tokens, g, h, lp, H, lse, dz, ldd, ws, n, None)


def d_forward(d=None, z=P, ld=40, t=None, loss=3 * P, lse=4 * P, ws=None, n=0):
    return mb.lib().mgrit_distill_forward(desc() if d is None else d, z, ld, teacher() if t is None else t, loss, lse, ws, n, None)


def d_backward(d=None, z=P, ld=40, t=None, lse=3 * P, g=4 * P, dz=5 * P, ldd=40):
    return mb.lib().mgrit_distill_backward(desc() if d is None else d, z, ld, teacher() if t is None else t, lse, g, dz, ldd, None)


def d_step(d=None, z=P, ld=40, t=None, g=3 * P, loss=4 * P, lse=5 * P, dz=7 * P, ldd=40, ws=None, n=0):
    return mb.lib().mgrit_distill_step(desc() if d is None else d, z, ld, teacher() if t is None else t, g, loss, lse, dz, ldd, ws, n, None)


@pytest.mark.parametrize("call", [forward, backward, step, d_forward, d_backward, d_step])
def test_descriptions_and_logits(call):
    for kw, status in BAD_DESCS:
        more = {} if call in (forward, d_forward) else dict(ldd=WIDE)
        assert call(desc(**kw), ld=WIDE, **more) == status, kw
    assert call(z=None) == INVALID and call(ld=39) == INVALID and call(ld=-40) == INVALID
    assert call(z=P + 2) == INVALID and call(desc(dtype=1), z=P + 1) == INVALID
    assert call(ld=1 << 41) == UNSUPPORTED
    if call not in (forward, d_forward):
        assert call(dz=None) == INVALID and call(ldd=39) == INVALID and call(dz=7 * P + 2) == INVALID
        assert call(dz=P, ldd=48) == INVALID                                           # in place at another place
    L = mb.lib()
    null = C.POINTER(mb.LogitsDesc)()
    assert L.mgrit_token_logprobs_workspace_bytes(null, 0, 0) == 0 and L.mgrit_distill_workspace_bytes(null, 1, 1) == 0


def test_forward_refusals():
    assert forward(tokens=None) == INVALID and forward(tokens=2 * P + 4) == INVALID and forward(desc(ids=0), tokens=2 * P + 2) == INVALID
    assert forward(tokens=None, lp=None, H=None, lse=None) == INVALID                  # nothing asked for
    assert forward(lp=3 * P + 1) == INVALID and forward(H=4 * P + 2) == INVALID and forward(lse=5 * P + 3) == INVALID
    assert forward(H=3 * P) == INVALID and forward(lse=3 * P) == INVALID and forward(lse=4 * P) == INVALID
    top = dict(k=5, ids=6 * P, top=7 * P)
    assert forward(**{**top, "k": -1}) == INVALID and forward(**{**top, "k": 41}) == INVALID
    assert forward(desc(cols=100), ld=100, **{**top, "k": 65}) == UNSUPPORTED
    assert forward(**{**top, "ids": None}) == INVALID and forward(**{**top, "top": None}) == INVALID
    assert forward(**{**top, "ids": 6 * P + 4}) == INVALID and forward(**{**top, "top": 7 * P + 2}) == INVALID
    assert forward(**{**top, "top": 6 * P}) == INVALID and forward(**{**top, "ids": 2 * P}) == INVALID and forward(**{**top, "top": 5 * P}) == INVALID
    none = desc(rows=0)
    assert forward(none, z=None, tokens=None) == OK and forward(none, k=3) == OK


def test_backward_and_step_refusals():
    assert backward(tokens=None) == INVALID and backward(lse=None) == INVALID and backward(g=None) == INVALID
    assert backward(tokens=2 * P + 4) == INVALID and backward(lse=3 * P + 2) == INVALID and backward(g=4 * P + 1) == INVALID
    assert backward(h=6 * P) == INVALID and backward(h=6 * P + 2, H=7 * P) == INVALID and backward(h=6 * P, H=7 * P + 2) == INVALID
    assert step(tokens=None) == INVALID and step(g=None) == INVALID and step(g=3 * P + 2) == INVALID and step(h=8 * P + 2) == INVALID
    assert step(lp=5 * P) == INVALID and step(lse=5 * P) == INVALID and step(lp=6 * P) == INVALID and step(lse=6 * P + 2) == INVALID
    none = desc(rows=0)
    assert backward(none, z=None, tokens=None, lse=None, g=None, dz=None) == OK and step(none, z=None, tokens=None, g=None, dz=None) == OK


def test_distill_refusals():
    for call in (d_forward, d_backward, d_step):
        assert call(t=teacher(kept=0)) == INVALID and call(t=teacher(kept=-2)) == INVALID and call(t=teacher(kept=257)) == UNSUPPORTED
        assert call(t=teacher(dtype=2)) == INVALID and call(t=teacher(ids=None)) == INVALID and call(t=teacher(logits=None)) == INVALID
        assert call(t=teacher(ids=20 * P + 4)) == INVALID and call(t=teacher(logits=21 * P + 2)) == INVALID and call(t=teacher(lse=22 * P + 2)) == INVALID
        assert call(t=C.POINTER(mb.Teacher)()) == INVALID
    assert d_forward(loss=None) == INVALID and d_forward(loss=3 * P + 2) == INVALID and d_forward(lse=3 * P) == INVALID and d_forward(lse=4 * P + 2) == INVALID
    assert d_backward(lse=None) == INVALID and d_backward(lse=3 * P + 2) == INVALID and d_backward(g=4 * P + 2) == INVALID
    assert d_step(loss=None) == INVALID and d_step(lse=4 * P) == INVALID and d_step(g=3 * P + 2) == INVALID
    empty = teacher(ids=None, logits=None)
    assert d_forward(desc(rows=0), z=None, t=empty, loss=None, lse=None) == OK and d_step(desc(rows=0), z=None, t=empty, loss=None, lse=None, dz=None) == OK


def test_workspaces():
    bf16, f32 = torch.bfloat16, torch.float32
    one, wide = desc(rows=1, cols=50257, dtype=1), desc(rows=4, cols=200001, dtype=1)
    top = dict(k=20, ids=6 * P, top=7 * P)
    need = mb.mgrit_token_logprobs_workspace_bytes(1, 50257, bf16, 20)
    assert need > mb.mgrit_token_logprobs_workspace_bytes(1, 50257, bf16) > 0
    assert forward(one, ld=50257, ws=8 * P, n=need - 1, **top) == SMALL
    assert forward(one, ld=50257, ws=None, n=need, **top) == INVALID and forward(one, ld=50257, ws=8 * P + 128, n=need, **top) == INVALID
    need = mb.mgrit_distill_workspace_bytes(1, 50257, bf16, 3)
    assert need > 0 and d_forward(one, ld=50257, ws=8 * P, n=need - 1) == SMALL and d_forward(one, ld=50257) == INVALID
    # a step needs one for rows that no block holds, and for few long ones
    assert mb.mgrit_token_logprobs_workspace_bytes(65, 131072, bf16, step=True) == 0 == mb.mgrit_distill_workspace_bytes(9000, 65536, f32, 3, step=True)
    assert mb.mgrit_token_logprobs_workspace_bytes(64, 131072, bf16, step=True) > 0 < mb.mgrit_distill_workspace_bytes(1, 65536, f32, 3, step=True)
    assert mb.mgrit_token_logprobs_workspace_bytes(1, 65536, bf16, step=True) == 0 == mb.mgrit_distill_workspace_bytes(1, 32768, f32, 3, step=True)
    need = mb.mgrit_token_logprobs_workspace_bytes(4, 200001, bf16, step=True)
    assert need > 0 and step(wide, ld=200001, ldd=200001, ws=8 * P, n=need - 1) == SMALL and step(wide, ld=200001, ldd=200001) == INVALID
    need = mb.mgrit_distill_workspace_bytes(4, 200001, bf16, 3, step=True)
    assert need > 0 and d_step(wide, ld=200001, ldd=200001, ws=8 * P, n=need - 1) == SMALL and d_step(wide, ld=200001, ldd=200001) == INVALID
    assert mb.mgrit_token_logprobs_workspace_bytes(9000, 65537, f32, step=True) > 0
    L = mb.lib()
    for kw, _ in BAD_DESCS:
        for s in (0, 1):
            assert L.mgrit_token_logprobs_workspace_bytes(desc(**kw), 0, s) == 0 and L.mgrit_distill_workspace_bytes(desc(**kw), 3, s) == 0
    assert L.mgrit_token_logprobs_workspace_bytes(one, 65, 0) == 0 and L.mgrit_distill_workspace_bytes(one, 257, 0) == 0
    assert mb.mgrit_token_logprobs_workspace_bytes(4096, 50257, bf16, 20) == 0                      # many rows need none
    assert mb.mgrit_token_logprobs_workspace_bytes(0, 50257, bf16, 20) == 0 == mb.mgrit_token_logprobs_workspace_bytes(0, 200001, bf16, step=True)
    with pytest.raises(ValueError, match="2\\^31 - 1"):
        mb.mgrit_token_logprobs_workspace_bytes(4, (1 << 32) + 40, f32)


@pytest.mark.parametrize("offset,ldd", [(39, 100), (61, 100), (1, 100), (-39, 100), (139, 100), (339, 100), (40, 101), (0, 101), (-300, 111)])
def test_gradients_that_lie_across_the_logits(offset, ldd):
    """4 rows of 40 fp32 elements at a distance of 100 (what is in order runs on the GPU)."""
    assert backward(z=8 * P, ld=100, dz=8 * P + 4 * offset, ldd=ldd) == INVALID
    assert step(z=8 * P, ld=100, dz=8 * P + 4 * offset, ldd=ldd) == INVALID
    assert d_backward(z=8 * P, ld=100, dz=8 * P + 4 * offset, ldd=ldd) == INVALID and d_step(z=8 * P, ld=100, dz=8 * P + 4 * offset, ldd=ldd) == INVALID


def test_gradients_that_lie_across_a_single_row():
    one = desc(rows=1)
    assert backward(one, z=8 * P, dz=8 * P + 4 * 39) == INVALID and backward(one, z=8 * P, dz=8 * P - 4 * 39) == INVALID
    assert backward(desc(dtype=1), z=8 * P, ld=100, dz=8 * P + 2 * 39, ldd=100) == INVALID and backward(desc(dtype=1), z=8 * P, ld=100, dz=8 * P + 2 * 61, ldd=100) == INVALID


def test_binding_refuses_what_the_library_cannot_see():
    z, t, g = torch.zeros(4, 40), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    ids, y = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3)
    for f in (lambda: mb.mgrit_token_logprobs_forward(z, t), lambda: mb.mgrit_token_logprobs_backward(z, t, g, g),
              lambda: mb.mgrit_token_logprobs_step(z, t, g), lambda: mb.mgrit_distill_forward(z, ids, y),
              lambda: mb.mgrit_distill_backward(z, ids, y, g), lambda: mb.mgrit_distill_step(z, ids, y)):
        with pytest.raises(ValueError, match="current device"):
            f()
    with pytest.raises(ValueError, match="expected a tensor"):
        mb.mgrit_token_logprobs_forward([1.0])


def test_steps_do_not_write_what_they_read():
    """A row's values are written while other wavefronts of the row still read its cotangents and its teacher."""
    for at in (-12, -4, 0, 4, 12):                         # 4 rows: 16 bytes each
        for out in ("lp", "H", "lse"):
            assert step(**{out: 30 * P + at}, g=30 * P) == INVALID
            assert step(**{out: 30 * P + at}, h=30 * P) == INVALID
        for out in ("loss", "lse"):
            assert d_step(**{out: 30 * P + at}, g=30 * P) == INVALID
            assert d_step(**{out: 30 * P + at}, t=teacher(lse=30 * P)) == INVALID
        assert step(lp=30 * P + at, H=30 * P) == INVALID and step(lse=30 * P + at, H=30 * P) == INVALID and step(lse=30 * P + at, lp=30 * P) == INVALID
        assert d_step(lse=30 * P + at, loss=30 * P) == INVALID


def test_workspace_query_of_no_count():
    f32 = torch.float32
    for k in ((1 << 32) + 5, -(1 << 32) + 5):
        with pytest.raises(ValueError, match="2\\^31 - 1"):
            mb.mgrit_token_logprobs_workspace_bytes(1, 50257, f32, k)


def test_no_rows_without_arrays():
    """A batch without rows has arrays without memory: nothing is asked for then, and nothing refused."""
    none = desc(rows=0)
    for tokens in (None, 2 * P):
        for k in (0, 3):
            assert forward(none, z=None, tokens=tokens, lp=None, H=None, lse=None, k=k) == OK
    for lse in (None, 22 * P):
        empty = teacher(ids=None, logits=None, lse=lse)
        assert d_forward(none, z=None, t=empty, loss=None, lse=None) == OK and d_backward(none, z=None, t=empty, lse=None, g=None, dz=None) == OK
        assert d_step(none, z=None, t=empty, g=None, loss=None, lse=None, dz=None) == OK
    assert step(none, z=None, tokens=None, g=None, lp=None, H=None, lse=None, dz=None) == OK
    assert forward(desc(rows=-1), z=None, tokens=None, lp=None, H=None, lse=None) == INVALID
    assert forward(tokens=None, lp=None, H=None, lse=None) == INVALID
