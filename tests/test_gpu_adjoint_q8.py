"""The adjoint from states that were kept in 8 bits: bit-identical to the adjoint on the unpacked states, with and without
the linearisation cache, and a whole training step with the last LayerNorm and kept rows."""
import types

import numpy as np
import pytest
import torch

from oracle import operators as oo
from paper_2601_09026_amd import binding as mb
from paper_2601_09026_amd import workloads as wls

from gpu_util import DeviceModel, dev

pytestmark = pytest.mark.gpu


def model(arch, dtype, d, layers, levels, batch=3, seq=21, mem=13):
    cf = 2 if levels > 1 else 1
    return wls.Workload("q8", arch, d, d // 32, 2 * d, batch, seq, mem if arch == wls.ARCH_CROSS else 0, layers, 1.0 / layers,
                        cf, levels, 2, dtype, 77)


@pytest.mark.parametrize("cache", [True, False])
@pytest.mark.parametrize("grads", [False, True])
@pytest.mark.parametrize("arch,dtype,d,layers,levels", [
    (wls.ARCH_ENCODER, wls.DTYPE_F32, 64, 16, 2), (wls.ARCH_CAUSAL, wls.DTYPE_BF16, 128, 12, 2),
    (wls.ARCH_CAUSAL, wls.DTYPE_BF16, 192, 16, 3), (wls.ARCH_CROSS, wls.DTYPE_BF16, 160, 8, 2),
    (wls.ARCH_CROSS, wls.DTYPE_F32, 96, 8, 1), (wls.ARCH_ENCODER, wls.DTYPE_BF16, 96, 9, 1)])
def test_as_on_the_unpacked_states(arch, dtype, d, layers, levels, grads, cache):
    print(f"[case] adjoint q8 arch={arch} dtype={dtype} d={d} N={layers} levels={levels} grads={grads} cache={cache}", flush=True)
    wl = model(arch, dtype, d, layers, levels)
    dm = DeviceModel(wl, weight_std=0.05, keep_host=False)
    opts = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    memory = dev(wls.cross_memory(wl)) if wl.mem_seq else None
    Z, _ = mb.mgrit_forward(dm.desc, opts, dev(wls.initial_state(wl)), dm.blocks, memory=memory)
    z8 = mb.mgrit_q8_pack(Z)
    lamN = dev(wls.terminal_adjoint(wl))

    def adjoint(states):
        g = [torch.zeros(mb.grad_layout(dm.desc).block_bytes, dtype=torch.uint8, device="cuda") for _ in range(wl.N)] if grads else None
        dmem = torch.zeros_like(memory) if grads and memory is not None else None
        lam, res = mb.mgrit_adjoint(dm.desc, opts, states, dm.blocks, lamN, memory=memory, dtheta=g, dmemory=dmem)
        return [lam, res, *(g or []), *([dmem] if dmem is not None else [])]

    mb.mgrit_set_adjoint_cache(cache)
    try:
        got, want, exact = adjoint(z8), adjoint(mb.mgrit_q8_unpack(z8)), adjoint(Z)
    finally:
        mb.mgrit_set_adjoint_cache(True)
    torch.cuda.synchronize()
    for p, q in zip(got, want):
        assert torch.equal(p, q)
    # and the rounding of the states is seen: not the adjoint about Z itself, but within a few steps of 1 / 127 of it
    assert not torch.equal(got[0][0], exact[0][0])
    assert float((got[0] - exact[0]).norm() / exact[0].norm()) < 0.02


@pytest.mark.parametrize("cache", [True, False])
@pytest.mark.parametrize("arch,dtype,d,layers,levels,batch,seq", [
    (wls.ARCH_ENCODER, wls.DTYPE_BF16, 40, 64, 3, 1, 1), (wls.ARCH_CAUSAL, wls.DTYPE_F32, 72, 8, 2, 2, 33),
    (wls.ARCH_CROSS, wls.DTYPE_F32, 8, 16, 2, 1, 5)])
def test_widths_that_are_not_whole_blocks(arch, dtype, d, layers, levels, batch, seq, cache):
    """Rows whose last block is filled up, a single token, and launches of many layers."""
    print(f"[case] adjoint q8, ragged blocks, arch={arch} dtype={dtype} d={d} N={layers} levels={levels} cache={cache}", flush=True)
    cf = 2 if levels > 1 else 1
    wl = wls.Workload("q8", arch, d, 1, 2 * d, batch, seq, 7 if arch == wls.ARCH_CROSS else 0, layers, 1.0 / layers, cf, levels, 2, dtype, 78)
    dm = DeviceModel(wl, weight_std=0.05, keep_host=False)
    opts = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    memory = dev(wls.cross_memory(wl)) if wl.mem_seq else None
    Z, _ = mb.mgrit_forward(dm.desc, opts, dev(wls.initial_state(wl)), dm.blocks, memory=memory)
    z8, lamN = mb.mgrit_q8_pack(Z), dev(wls.terminal_adjoint(wl))
    mb.mgrit_set_adjoint_cache(cache)
    try:
        runs = []
        for states in (z8, mb.mgrit_q8_unpack(z8)):
            g = [torch.zeros(mb.grad_layout(dm.desc).block_bytes, dtype=torch.uint8, device="cuda") for _ in range(wl.N)]
            lam, res = mb.mgrit_adjoint(dm.desc, opts, states, dm.blocks, lamN, memory=memory, dtheta=g)
            runs.append([lam, res, *g])
    finally:
        mb.mgrit_set_adjoint_cache(True)
    for p, q in zip(*runs):
        assert torch.equal(p, q)


def test_workspaces_and_refusals():
    print("[case] adjoint q8 refusals", flush=True)
    wl = model(wls.ARCH_ENCODER, wls.DTYPE_F32, 64, 8, 2)
    dm = DeviceModel(wl, keep_host=False)
    opts = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    Z, _ = mb.mgrit_forward(dm.desc, opts, dev(wls.initial_state(wl)), dm.blocks)
    z8, lamN = mb.mgrit_q8_pack(Z), dev(wls.terminal_adjoint(wl))
    with pytest.raises(ValueError, match="8-bit rows of shape"):
        mb.mgrit_adjoint(dm.desc, opts, z8[:8], dm.blocks, lamN)
    with pytest.raises(ValueError, match="linearised"):
        mb.mgrit_adjoint(dm.desc, opts, z8, dm.blocks, lamN, linearised=True)
    short = torch.empty(mb.mgrit_workspace_bytes(dm.desc, opts, 1), dtype=torch.uint8, device="cuda")
    with pytest.raises(mb.MgritError, match="workspace too small"):
        mb.mgrit_adjoint(dm.desc, opts, z8, dm.blocks, lamN, workspace=short)


def test_a_training_step_with_kept_rows():
    """Forward solve, last LayerNorm with copies in 8 bits, a linear head, and back: head gradient and LayerNorm backward
    from the kept rows, adjoint from the kept states.  Each stage against the float64 definition on its own inputs; the
    tolerances are those of an fp32 stage (1e-6 of the norm)."""
    print("[case] training step with kept rows", flush=True)
    wl = model(wls.ARCH_CAUSAL, wls.DTYPE_F32, 96, 8, 2)
    dm = DeviceModel(wl, weight_std=0.05, keep_host=False)
    opts = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    rng = np.random.default_rng(4)
    W, gamma, beta = (dev(rng.standard_normal(s)) for s in ((50, 96), 96, 96))
    Z, _ = mb.mgrit_forward(dm.desc, opts, dev(wls.initial_state(wl)), dm.blocks)
    kept_y = mb.q8_empty((wl.tokens, 96))
    y, mean, rstd = mb.mgrit_layer_norm_forward(Z[-1], gamma, beta, y_q8=kept_y)
    kept_z = mb.mgrit_q8_pack(Z)
    dlogits = dev(rng.standard_normal((wl.tokens, 50)))
    dW, db = mb.mgrit_q8_weight_grad(dlogits, kept_y)
    lamN, dgamma, dbeta = mb.mgrit_layer_norm_backward(dlogits @ W, kept_z[-1], gamma, mean, rstd)
    lam, _ = mb.mgrit_adjoint(dm.desc, opts, kept_z, dm.blocks, lamN)
    n = lambda t: t.double().cpu().numpy()  # noqa: E731
    def near(got, ref):
        assert np.linalg.norm(n(got) - ref) <= 1e-6 * np.linalg.norm(ref)
    ry, rm, rr = oo.norm_forward(n(Z[-1]), n(gamma), n(beta), 1e-5)
    near(y, ry)
    y8 = oo.q8_unpack(*oo.q8_pack(n(y)), 96)
    rW, rb = oo.weight_grad(n(dlogits), y8)
    near(dW, rW)
    near(db, rb)
    rx, rg, rbeta = oo.norm_backward(n(dlogits @ W), oo.q8_unpack(*oo.q8_pack(n(Z[-1])), 96), n(gamma), n(mean), n(rstd))
    near(lamN, rx)
    near(dgamma, rg)
    near(dbeta, rbeta)
    ref, _ = mb.mgrit_adjoint(dm.desc, opts, mb.mgrit_q8_unpack(kept_z), dm.blocks, lamN)
    assert torch.equal(lam, ref)


@pytest.mark.parametrize("cache", [True, False])
def test_captured_calls_replay_bit_identically(cache):
    print(f"[case] captured adjoint q8 cache={cache}", flush=True)
    wl = model(wls.ARCH_CAUSAL, wls.DTYPE_BF16, 128, 8, 2)
    dm = DeviceModel(wl, weight_std=0.05, keep_host=False)
    opts = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    Z, _ = mb.mgrit_forward(dm.desc, opts, dev(wls.initial_state(wl)), dm.blocks)
    lamN, z8 = dev(wls.terminal_adjoint(wl)), mb.q8_empty(Z.shape)
    mb.mgrit_set_adjoint_cache(cache)
    try:
        ws = torch.empty(mb.mgrit_adjoint_q8_workspace_bytes(dm.desc, opts, 1), dtype=torch.uint8, device="cuda")
        def run():
            return mb.mgrit_adjoint(dm.desc, opts, mb.mgrit_q8_pack(Z, out=z8), dm.blocks, lamN, workspace=ws)
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = run()
        for rep in range(3):
            for t in (*got, z8.q, z8.scale):
                t.fill_(rep + 1)
            ws.fill_(255)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for p, q in zip(got, want):
                assert torch.equal(p, q), f"replay {rep}"
    finally:
        mb.mgrit_set_adjoint_cache(True)


@pytest.mark.parametrize("cache", [True, False])
@pytest.mark.parametrize("form", ["kept", "unpacked"])
def test_another_stream_than_the_current_one(form, cache):
    """stream=: outputs and workspace are the call's own and belong to its stream, operands are kept for it.  First the other
    stream is held up, so that the call has returned, its temporaries are gone and their memory is asked for again before
    it runs; then the current one, so that nothing of the call may wait there."""
    print(f"[case] adjoint on another stream, {form}, cache={cache}", flush=True)
    wl = model(wls.ARCH_CROSS, wls.DTYPE_F32, 96, 8, 2)
    dm = DeviceModel(wl, weight_std=0.05, keep_host=False)
    opts = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    memory, lamN = dev(wls.cross_memory(wl)), dev(wls.terminal_adjoint(wl))
    Z, _ = mb.mgrit_forward(dm.desc, opts, dev(wls.initial_state(wl)), dm.blocks, memory=memory)
    z8 = mb.mgrit_q8_pack(Z)
    copy = lambda t: mb.Q8Rows(t.q.clone(), t.scale.clone(), t.cols) if isinstance(t, mb.Q8Rows) else t.clone()  # noqa: E731
    states = z8 if form == "kept" else Z

    def adjoint(stream):
        """On copies of the operands that go when this returns."""
        g = [torch.zeros(mb.grad_layout(dm.desc).block_bytes, dtype=torch.uint8, device="cuda") for _ in range(wl.N)]
        args = copy(states), [copy(b) for b in dm.blocks], copy(lamN), copy(memory)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                torch.cuda._sleep(100_000_000)
        lam, res = mb.mgrit_adjoint(dm.desc, opts, *args[:3], memory=args[3], dtheta=g, stream=stream)
        return [lam, res, *g]

    mb.mgrit_set_adjoint_cache(cache)
    try:
        want = adjoint(None)
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        s = torch.cuda.Stream()
        need = (mb.mgrit_adjoint_q8_workspace_bytes if form == "kept" else mb.mgrit_workspace_bytes)(dm.desc, opts, 2)
        got = adjoint(s)
        sizes = [need, *[t.numel() * t.element_size() for t in (Z, lamN, memory, z8.q, z8.scale, *dm.blocks)]]
        junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
        torch.cuda.synchronize()
        assert all(bool((j == 255).all()) for j in junk)
        for p, q in zip(got, want):
            assert torch.equal(p, q)
        torch.cuda._sleep(100_000_000)                     # the current stream
        lam, res = mb.mgrit_adjoint(dm.desc, opts, states, dm.blocks, lamN, memory=memory, stream=s)
        s.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(lam, want[0]) and torch.equal(res, want[1])
    finally:
        mb.mgrit_set_adjoint_cache(True)


def test_adjoint_on_a_stream_of_another_device_is_refused():
    print("[case] adjoint on a stream of another device", flush=True)
    wl = model(wls.ARCH_ENCODER, wls.DTYPE_F32, 64, 8, 2)
    dm = DeviceModel(wl, keep_host=False)
    opts = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters)
    Z, lamN = dev(np.zeros((wl.N + 1, wl.tokens, wl.d_model))), dev(wls.terminal_adjoint(wl))
    other = types.SimpleNamespace(device_index=torch.cuda.current_device() + 1, cuda_stream=0)
    for states in (Z, mb.mgrit_q8_pack(Z)):
        with pytest.raises(ValueError, match="current device"):
            mb.mgrit_adjoint(dm.desc, opts, states, dm.blocks, lamN, stream=other)
