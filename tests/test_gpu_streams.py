"""stream=: every solve and layer step on another stream than the current one.  What the binding allocates belongs to that
stream and operands are kept for it, so that nothing is handed out again before the call has run; results are those of the
current stream, bit for bit."""
import types

import pytest
import torch

from paper_2601_09026_amd import binding as mb
from paper_2601_09026_amd import workloads as wls

from gpu_util import DeviceModel, dev
from test_gpu_stacked import stacked

pytestmark = pytest.mark.gpu


def copies(*operands):
    return [[t.clone() for t in v] if isinstance(v, list) else v.clone() for v in operands]


def jobs():
    """name -> (sizes in bytes of what a call allocates or is given, call(stream) on copies of its operands)."""
    wl = wls.Workload("streams", wls.ARCH_ENCODER, 96, 3, 192, 3, 21, 0, 8, 0.125, 2, 2, 2, wls.DTYPE_F32, 31)
    dm = DeviceModel(wl, n_layers=10, weight_std=0.05, keep_host=False)
    opts, buf = mb.mgrit_opts(wl.N, wl.h, wl.cf, wl.levels, wl.iters), mb.BufferOpts(1, 1, 1.0)
    Z0, lamN, theta = dev(wls.initial_state(wl)), dev(wls.terminal_adjoint(wl)), dm.blocks[:wl.N]
    Z, _ = mb.mgrit_forward(dm.desc, opts, Z0, theta)
    Zb, _ = mb.mgrit_forward_buffered(dm.desc, opts, buf, Z0, dm.blocks)
    sw = stacked(n_enc=4, n_dec=4, cf=2)
    dd = mb.model_desc(sw.dec)
    de = mb.encoder_desc(dd)
    sopts = mb.mgrit_opts(sw.N, sw.dec.h, sw.dec.cf, sw.dec.levels, sw.dec.iters)
    blocks = [mb.pack_theta(de if n < sw.n_enc else dd, wls.stacked_layer_params(sw, n, 0.05)) for n in range(sw.N)]
    S0 = dev(wls.stacked_initial_state(sw))
    Zs, _ = mb.mgrit_forward_stacked(dd, sopts, sw.n_enc, S0, blocks)
    grads = lambda desc, n: [torch.zeros(mb.grad_layout(desc).block_bytes, dtype=torch.uint8, device="cuda") for _ in range(n)]  # noqa: E731
    lin_ws = mb.mgrit_workspace_bytes(dm.desc, opts, 1)

    def pair(stream, Z0, theta, lamN, ws):
        Z, rz = mb.mgrit_forward(dm.desc, opts, Z0, theta, stream=stream, adjoint_workspace=ws)
        return [Z, rz, *mb.mgrit_adjoint(dm.desc, opts, Z, theta, lamN, stream=stream, workspace=ws, linearised=True)]

    def adjoint_buffered(stream, Z, theta, lamN, g):
        return [*mb.mgrit_adjoint_buffered(dm.desc, opts, buf, Z, theta, lamN, dtheta=g, stream=stream), *g]

    def adjoint_stacked(stream, Z, theta, lamN, g):
        return [*mb.mgrit_adjoint_stacked(dd, sopts, sw.n_enc, Z, theta, lamN, dtheta=g, stream=stream), *g]

    def steps(entry):
        def call(stream, inputs, theta, rhs, out):
            return entry(dm.desc, False, inputs, out, theta, 0.5, rhs=rhs, stream=stream)
        return call

    states = [Z[n].contiguous() for n in range(4)]
    all_jobs = {
        "forward": (mb.mgrit_workspace_bytes(dm.desc, opts, 0), lambda st, *a: list(mb.mgrit_forward(dm.desc, opts, *a, stream=st)), (Z0, theta)),
        "linearised pair": (mb.mgrit_linearising_workspace_bytes(dm.desc, opts), pair,
                            (Z0, theta, lamN, torch.zeros(lin_ws, dtype=torch.uint8, device="cuda"))),
        "buffered forward": (mb.mgrit_buffered_workspace_bytes(dm.desc, opts, buf, 0),
                             lambda st, *a: list(mb.mgrit_forward_buffered(dm.desc, opts, buf, *a, stream=st)), (Z0, dm.blocks)),
        "buffered adjoint": (mb.mgrit_buffered_workspace_bytes(dm.desc, opts, buf, 2), adjoint_buffered,
                             (Zb, dm.blocks, lamN, grads(dm.desc, 10))),
        "stacked forward": (mb.mgrit_stacked_workspace_bytes(dd, sopts, sw.n_enc, 0),
                            lambda st, *a: list(mb.mgrit_forward_stacked(dd, sopts, sw.n_enc, *a, stream=st)), (S0, blocks)),
        "stacked adjoint": (mb.mgrit_stacked_workspace_bytes(dd, sopts, sw.n_enc, 2), adjoint_stacked,
                            (Zs, blocks, torch.ones_like(S0), [*grads(de, sw.n_enc), *grads(dd, sw.N - sw.n_enc)])),
        "layer step": (mb.mgrit_layer_step_workspace_bytes(dm.desc, False, 4), steps(mb.layer_step_batched),
                       (states, theta[:4], states, [torch.zeros_like(t) for t in states])),
        "layer step, fixed array": (256, steps(mb.layer_step_batched_static),
                                    (states, theta[:4], states, [torch.zeros_like(t) for t in states])),
    }
    return all_jobs


NAMES = ["forward", "linearised pair", "buffered forward", "buffered adjoint", "stacked forward", "stacked adjoint", "layer step",
         "layer step, fixed array"]


def flat(operands):
    return [t for v in operands for t in (v if isinstance(v, list) else [v])]


@pytest.mark.parametrize("name", NAMES)
def test_another_stream_than_the_current_one(name):
    """First the other stream is held up, so that the call has returned, its temporaries are gone and their memory is asked for
    again before it runs; then the current one, so that nothing of the call may wait there."""
    print(f"[case] another stream: {name}", flush=True)
    all_jobs = jobs()
    assert list(all_jobs) == NAMES
    need, call, operands = all_jobs[name]

    def run(stream):
        args = copies(*operands)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                torch.cuda._sleep(100_000_000)
        return call(stream, *args)

    want = run(None)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    s = torch.cuda.Stream()
    got = run(s)
    sizes = [need, *[t.numel() * t.element_size() for t in flat(operands)]]
    junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda.synchronize()
    assert all(bool((j == 255).all()) for j in junk)
    for p, q in zip(got, want):
        assert torch.equal(p, q)
    args = copies(*operands)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                         # the current stream
    got = call(s, *args)
    s.synchronize()
    torch.cuda.synchronize()
    for p, q in zip(got, want):
        assert torch.equal(p, q)


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device_is_refused(name):
    print(f"[case] a stream of another device: {name}", flush=True)
    _, call, operands = jobs()[name]
    other = types.SimpleNamespace(device_index=torch.cuda.current_device() + 1, cuda_stream=0)
    with pytest.raises(ValueError, match="current device"):
        call(other, *copies(*operands))
