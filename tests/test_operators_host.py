"""What the operators around the solves refuse, before anything is enqueued: null and misaligned pointers, sizes, types,
strides, workspaces; and host-side queries.  Needs no GPU: the pointers are numbers that are never followed."""
import ctypes as C

import pytest
import torch

from paper_2601_09026_amd import binding as mb
from paper_2601_09026_amd import workloads as wls

INVALID, UNSUPPORTED, SMALL = mb.MGRIT_INVALID_ARG, mb.MGRIT_UNSUPPORTED, mb.MGRIT_WORKSPACE_TOO_SMALL
P = 1 << 20                                               # an aligned address


def test_blocks():
    assert [mb.mgrit_q8_blocks(c) for c in (0, -3, 1, 31, 32, 33, 768)] == [0, 0, 1, 1, 1, 2, 24]


@pytest.mark.parametrize("entry", ["mgrit_q8_pack", "mgrit_q8_unpack"])
def test_q8_refusals(entry):
    def call(rows=4, cols=40, dtype=0, x=P, stride=40, q=2 * P, scale=3 * P):
        f = getattr(mb.lib(), entry)
        return f(rows, cols, dtype, x, stride, q, scale, None) if entry.endswith("_pack") else \
            f(rows, cols, dtype, q, scale, x, stride, None)
    assert call(rows=-1) == INVALID and call(cols=0) == INVALID and call(dtype=2) == INVALID and call(dtype=-1) == INVALID
    assert call(x=None) == INVALID and call(q=None) == INVALID and call(scale=None) == INVALID
    assert call(stride=39) == INVALID and call(stride=-40) == INVALID
    assert call(x=P + 2) == INVALID and call(x=P + 1, dtype=1) == INVALID and call(q=2 * P + 8) == INVALID
    assert call(rows=1 << 41) == UNSUPPORTED and call(stride=1 << 41) == UNSUPPORTED
    assert call(rows=0, x=None, q=None, scale=None) == mb.MGRIT_OK


def norm(rows=4, cols=40, x_dtype=0, y_dtype=0, eps=1e-5):
    return mb.NormDesc(rows, cols, x_dtype, y_dtype, eps)


BAD_DESCS = [(dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(x_dtype=3), INVALID), (dict(y_dtype=-1), INVALID),
             (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
             (dict(cols=16385), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED)]


def test_norm_forward_refusals():
    def call(desc=None, x=P, ldx=40, gamma=2 * P, beta=3 * P, y=4 * P, ldy=40, mean=5 * P, rstd=6 * P, xq=None, xs=None,
             yq=None, ys=None):
        d = norm() if desc is None else desc
        return mb.lib().mgrit_layer_norm_forward(C.byref(d), x, ldx, gamma, beta, y, ldy, mean, rstd, xq, xs, yq, ys, None)
    for kw, status in BAD_DESCS:
        assert call(norm(**kw), ldx=1 << 15, ldy=1 << 15) == status, kw
    assert mb.lib().mgrit_layer_norm_forward(None, P, 40, None, None, P, 40, None, None, None, None, None, None, None) == INVALID
    assert call(x=None) == INVALID and call(y=None) == INVALID and call(ldx=39) == INVALID and call(ldy=39) == INVALID
    assert call(gamma=2 * P + 2) == INVALID and call(mean=5 * P + 1) == INVALID and call(x=P + 2) == INVALID
    assert call(xq=7 * P) == INVALID and call(xs=7 * P) == INVALID and call(yq=7 * P) == INVALID and call(ys=7 * P) == INVALID
    assert call(xq=7 * P + 8, xs=8 * P) == INVALID
    assert call(y=P, ldy=48) == INVALID and call(norm(y_dtype=1), y=P) == INVALID          # in place at another place
    assert call(norm(rows=0), x=None, y=None, gamma=None, beta=None, mean=None, rstd=None) == mb.MGRIT_OK
    # one array for two results
    assert call(rstd=5 * P) == INVALID
    assert call(xq=7 * P, xs=8 * P, yq=7 * P, ys=9 * P) == INVALID and call(xq=7 * P, xs=8 * P, yq=9 * P, ys=8 * P) == INVALID


def test_norm_backward_refusals():
    def call(desc=None, dy=P, lddy=40, x=2 * P, ldx=40, xq=None, xs=None, gamma=3 * P, mean=4 * P, rstd=5 * P, dx=6 * P,
             lddx=40, dg=7 * P, db=8 * P, ws=9 * P, n=1 << 20):
        d = norm() if desc is None else desc
        return mb.lib().mgrit_layer_norm_backward(C.byref(d), dy, lddy, x, ldx, xq, xs, gamma, mean, rstd, dx, lddx, dg,
                                                  db, ws, n, None)
    for kw, status in BAD_DESCS:
        assert call(norm(**kw), lddy=1 << 15, ldx=1 << 15, lddx=1 << 15) == status, kw
        assert mb.lib().mgrit_layer_norm_backward_workspace_bytes(C.byref(norm(**kw))) == 0
    assert call(x=None) == INVALID                                                        # neither form of x
    assert call(xq=10 * P, xs=11 * P) == INVALID                                          # both
    assert call(x=None, xq=10 * P) == INVALID and call(x=None, xq=10 * P + 4, xs=11 * P) == INVALID
    assert call(dy=None) == INVALID and call(mean=None) == INVALID and call(rstd=None) == INVALID
    assert call(lddy=39) == INVALID and call(ldx=39) == INVALID and call(lddx=39) == INVALID
    assert call(dx=None, dg=None, db=None) == INVALID
    assert call(dx=P) == INVALID and call(dx=2 * P) == INVALID                            # dx over dy, over x
    assert call(dg=7 * P + 2) == INVALID and call(db=8 * P + 1) == INVALID and call(db=7 * P) == INVALID
    many = norm(rows=5000)
    need = mb.lib().mgrit_layer_norm_backward_workspace_bytes(C.byref(many))
    assert need > 0 and call(many, n=need - 1) == SMALL
    assert call(many, ws=None) == INVALID and call(many, ws=9 * P + 128) == INVALID
    assert call(norm(rows=0), dy=None, x=None, mean=None, rstd=None, dx=None, dg=None, db=None) == INVALID


def test_weight_grad_refusals():
    def call(rows=4, m=24, k=40, dtype=0, dy=P, lddy=24, xq=2 * P, xs=3 * P, scale=1.0, dW=4 * P, db=5 * P, ws=6 * P,
             n=1 << 24):
        return mb.lib().mgrit_q8_weight_grad(rows, m, k, dtype, dy, lddy, xq, xs, scale, dW, db, ws, n, None)
    assert call(rows=-1) == INVALID and call(m=0) == INVALID and call(k=0) == INVALID and call(dtype=2) == INVALID
    assert call(dy=None) == INVALID and call(xq=None) == INVALID and call(xs=None) == INVALID and call(dW=None) == INVALID
    assert call(lddy=23) == INVALID and call(dy=P + 2) == INVALID and call(xq=2 * P + 8) == INVALID
    assert call(dW=4 * P + 2) == INVALID and call(db=5 * P + 1) == INVALID
    assert call(scale=float("inf")) == INVALID and call(scale=float("nan")) == INVALID
    assert call(m=1 << 16, k=1 << 16, lddy=1 << 16) == UNSUPPORTED and call(rows=1 << 31) == UNSUPPORTED
    assert call(m=(1 << 24) + 1, k=1, lddy=1 << 25) == UNSUPPORTED and call(lddy=(1 << 24) + 1) == UNSUPPORTED
    need = mb.mgrit_q8_weight_grad_workspace_bytes(8192, 64, 64, torch.float32)
    assert need > 0 and call(rows=8192, m=64, k=64, lddy=64, n=need - 1) == SMALL
    assert call(rows=8192, m=64, k=64, lddy=64, ws=None) == INVALID and call(rows=8192, m=64, k=64, lddy=64, ws=6 * P + 64) == INVALID
    assert mb.lib().mgrit_q8_weight_grad_workspace_bytes(-1, 4, 4, 0) == 0
    most = (1 << 31) - 256
    assert call(rows=most + 1, m=1, k=1) == UNSUPPORTED and mb.mgrit_q8_weight_grad_workspace_bytes(most + 1, 1, 1, torch.float32) == 0
    assert mb.mgrit_q8_weight_grad_workspace_bytes(most, 1, 1, torch.float32) > 0


def test_workspace_sizes_do_not_fall_with_the_rows():
    sizes = [mb.mgrit_layer_norm_backward_workspace_bytes(r, 768) for r in (0, 1, 64, 4096, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] == 0 < sizes[-1]


def test_adjoint_q8_host_side():
    wl = wls.named_workloads()["tiny_encoder"]
    desc, opts = mb.model_desc(wl), mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    L = mb.lib()
    states = 4 * wl.N * wl.tokens * wl.d_model
    for mode in (1, 2):
        plain, q8 = mb.mgrit_workspace_bytes(desc, opts, mode), mb.mgrit_adjoint_q8_workspace_bytes(desc, opts, mode)
        assert plain + states <= q8 <= plain + states + 1024
        mb.mgrit_set_adjoint_cache(False)
        try:                                              # a chunk's states instead of all: less than one more set
            lean = mb.mgrit_adjoint_q8_workspace_bytes(desc, opts, mode)
            assert mb.mgrit_workspace_bytes(desc, opts, mode) < lean < q8
        finally:
            mb.mgrit_set_adjoint_cache(True)
    assert mb.mgrit_adjoint_q8_workspace_bytes(desc, opts, 0) == 0 and mb.mgrit_adjoint_q8_workspace_bytes(desc, opts, 3) == 0
    theta = (C.c_void_p * wl.N)(*[P] * wl.N)
    def call(z=P, s=2 * P, lam=3 * P, out=4 * P, ws=5 * P, n=1 << 40):
        return L.mgrit_adjoint_q8(C.byref(desc), C.byref(opts), z, s, theta, None, lam, out, None, None, None, ws, n, None)
    assert call(z=None) == INVALID and call(s=None) == INVALID and call(z=P + 8) == INVALID and call(lam=None) == INVALID
    assert call(out=None) == INVALID and call(ws=None) == INVALID
    assert call(n=mb.mgrit_workspace_bytes(desc, opts, 1)) == SMALL


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 40)
    for f in (lambda: mb.mgrit_q8_pack(x), lambda: mb.mgrit_layer_norm_forward(x),
              lambda: mb.mgrit_q8_unpack(mb.q8_empty((4, 40), "cpu")),
              lambda: mb.mgrit_layer_norm_backward(x, x, None, x[:, 0], x[:, 0]),
              lambda: mb.mgrit_q8_weight_grad(x, mb.q8_empty((4, 40), "cpu"))):
        with pytest.raises(ValueError, match="current device"):
            f()
    q, s = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8)
    assert mb.Q8Rows(q, s, 40).shape == (4, 40) and mb.Q8Rows(q, s, 64)[1:3].shape == (2, 64)
    for bad in ((q, s, 32), (q, s, 65), (q.to(torch.uint8), s, 40), (q, s.to(torch.int8), 40), (q[:3], s, 40), (q, s, 0)):
        with pytest.raises(ValueError):
            mb.Q8Rows(*bad)
    with pytest.raises(IndexError):
        mb.Q8Rows(q, s, 40)[0, 1]


def test_binding_refuses_lengths_of_more_than_32_bits():
    """The header's row lengths have 32 bits; a longer one is refused and not cut."""
    n = (1 << 32) + 40
    for f in (lambda: mb.mgrit_q8_blocks(n), lambda: mb.q8_empty((2, n), "meta"),
              lambda: mb.mgrit_layer_norm_backward_workspace_bytes(5000, n),
              lambda: mb.mgrit_q8_weight_grad_workspace_bytes(8, n, 4, torch.float32),
              lambda: mb.mgrit_q8_weight_grad_workspace_bytes(8, 4, n, torch.float32),
              lambda: mb.Q8Rows(torch.empty((1, n + 24), dtype=torch.int8, device="meta"),
                                torch.empty((1, n // 32 + 1), dtype=torch.uint8, device="meta"), n)):
        with pytest.raises(ValueError, match="2\\^31 - 1|expected int8"):
            f()


def test_other_adjoints_refuse_kept_states():
    wl = wls.named_workloads()["tiny_encoder"]
    desc, opts = mb.model_desc(wl), mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    z8 = mb.q8_empty((wl.N + 1, wl.tokens, wl.d_model), "cpu")
    lam = torch.zeros(wl.tokens, wl.d_model)
    with pytest.raises(ValueError, match="expected a tensor, got Q8Rows"):
        mb.mgrit_adjoint_buffered(desc, opts, mb.BufferOpts(0, 0, 0.0), z8, [lam] * wl.N, lam)
    with pytest.raises(ValueError, match="expected a tensor, got Q8Rows"):
        mb.mgrit_forward(desc, opts, z8, [lam] * wl.N)


def test_binding_names_what_is_of_the_wrong_kind():
    x, x8 = torch.zeros(4, 40), mb.q8_empty((4, 40), "cpu")
    for f, kind in ((lambda: mb.mgrit_q8_pack(x8), "tensor, got Q8Rows"), (lambda: mb.mgrit_q8_unpack(x), "Q8Rows, got Tensor"),
                    (lambda: mb.mgrit_layer_norm_forward(x8), "tensor, got Q8Rows"),
                    (lambda: mb.mgrit_layer_norm_backward(x8, x, None, x[:, 0], x[:, 0]), "tensor, got Q8Rows"),
                    (lambda: mb.mgrit_q8_weight_grad(x8, x8), "tensor, got Q8Rows")):
        with pytest.raises(ValueError, match=kind):
            f()


def test_weight_grad_refuses_one_array_for_two_results():
    def call(dW, db, rows=4):
        return mb.lib().mgrit_q8_weight_grad(rows, 24, 1, 0, P, 24, 2 * P, 3 * P, 1.0, dW, db, 6 * P, 1 << 24, None)
    # (one input feature: dW and db have the same size)
    assert call(4 * P, 4 * P) == INVALID and call(4 * P, 4 * P, rows=0) == INVALID
