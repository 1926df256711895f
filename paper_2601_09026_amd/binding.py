"""Thin ctypes binding over the C-ABI HIP library (argument marshalling only).

Function names mirror include/mgrit.h.  PyTorch is used for device memory and
streams; every computation happens inside the library's kernels.  There is no
CPU fallback: if the shared library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmgrit_hip.so")

MGRIT_OK = 0
MGRIT_INVALID_ARG, MGRIT_UNSUPPORTED, MGRIT_WORKSPACE_TOO_SMALL, MGRIT_HIP_ERROR = -1, -2, -3, -4
P_NAMES = ["ln1_g", "ln1_b", "bqkv", "bo", "ln2_g", "ln2_b", "b1", "b2", "ln3_g", "ln3_b", "bq_c",
           "bkv_c", "bo_c", "Wqkv", "Wo", "W1", "W2", "Wq_c", "Wkv_c", "Wo_c"]
P_COUNT = len(P_NAMES)


class Indicator(C.Structure):
    """mgrit_indicator: the host-side inexactness controller (plain data)."""
    _fields_ = [("iters", C.c_int32), ("probe_every", C.c_int32), ("mitigation", C.c_int32),
                ("max_iters", C.c_int32), ("threshold", C.c_float), ("last_factor", C.c_float),
                ("batch", C.c_int64), ("serial", C.c_int32), ("probing", C.c_int32), ("failures", C.c_int32),
                ("reserved", C.c_int32)]


MITIGATE_SERIAL, MITIGATE_MORE_ITERATIONS = 0, 1


class BufferOpts(C.Structure):
    _fields_ = [("n_open", C.c_int32), ("n_close", C.c_int32), ("h_buffer", C.c_float)]


class ModelDesc(C.Structure):
    _fields_ = [("arch", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("d_ff", C.c_int32),
                ("batch", C.c_int32), ("seq", C.c_int32), ("mem_seq", C.c_int32), ("dtype", C.c_int32),
                ("ln_eps", C.c_float)]


class Opts(C.Structure):
    _fields_ = [("N", C.c_int32), ("h", C.c_float), ("cf", C.c_int32), ("levels", C.c_int32),
                ("iters", C.c_int32), ("relax", C.c_int32), ("init_guess", C.c_int32)]


class NormDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32),
                ("eps", C.c_float)]


class ThetaLayout(C.Structure):
    _fields_ = [("block_bytes", C.c_int64), ("offset", C.c_int64 * P_COUNT), ("rows", C.c_int32 * P_COUNT),
                ("cols", C.c_int32 * P_COUNT), ("elem_bytes", C.c_int32 * P_COUNT)]


class MgritError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().mgrit_status_string(status).decode()
        hip = lib().mgrit_last_hip_error() if status == -4 else 0
        super().__init__(f"{where}: {msg} (status {status}" + (f", hipError {hip})" if hip else ")"))


_lib = None


def lib() -> C.CDLL:
    """Load the HIP library (built by `python -m paper_2601_09026_amd.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2601_09026_amd.build` (no CPU fallback exists)")
        L = C.CDLL(LIB_PATH)
        vp, vpp = C.c_void_p, C.POINTER(C.c_void_p)
        L.mgrit_theta_layout.argtypes = [C.POINTER(ModelDesc), C.POINTER(ThetaLayout)]
        L.mgrit_theta_layout.restype = C.c_int
        L.mgrit_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.c_int]
        L.mgrit_workspace_bytes.restype = C.c_size_t
        L.mgrit_linearising_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts)]
        L.mgrit_linearising_workspace_bytes.restype = C.c_size_t
        L.mgrit_layer_step_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.c_int, C.c_int]
        L.mgrit_layer_step_workspace_bytes.restype = C.c_size_t
        L.mgrit_step_evaluations.argtypes = [C.POINTER(Opts)]
        L.mgrit_step_evaluations.restype = C.c_int64
        L.mgrit_measure_mfma_ceiling.argtypes = [C.c_void_p, C.c_size_t, C.c_int, C.POINTER(C.c_double), C.c_void_p]
        L.mgrit_measure_mfma_ceiling.restype = C.c_int
        L.mgrit_measure_copy_ceiling.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.POINTER(C.c_double), C.c_void_p]
        L.mgrit_measure_copy_ceiling.restype = C.c_int
        L.mgrit_step_depth.argtypes = [C.POINTER(Opts)]
        L.mgrit_step_depth.restype = C.c_int64
        L.mgrit_forward.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), vp, vpp, vp, vp, vp, vp,
                                    C.c_size_t, vp]
        L.mgrit_forward.restype = C.c_int
        L.mgrit_adjoint.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), vp, vpp, vp, vp, vp, vp, vpp, vp,
                                    vp, C.c_size_t, vp]
        L.mgrit_adjoint.restype = C.c_int
        L.mgrit_forward_linearising.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), vp, vpp, vp, vp, vp, vp,
                                                C.c_size_t, vp, C.c_size_t, C.c_int, vp]
        L.mgrit_forward_linearising.restype = C.c_int
        L.mgrit_adjoint_linearised.argtypes = L.mgrit_adjoint.argtypes
        L.mgrit_adjoint_linearised.restype = C.c_int
        L.mgrit_adjoint_q8_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.c_int]
        L.mgrit_adjoint_q8_workspace_bytes.restype = C.c_size_t
        L.mgrit_adjoint_q8.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), vp, vp, vpp, vp, vp, vp, vp, vpp, vp,
                                       vp, C.c_size_t, vp]
        L.mgrit_adjoint_q8.restype = C.c_int
        i64, i32, nd = C.c_int64, C.c_int32, C.POINTER(NormDesc)
        L.mgrit_q8_blocks.argtypes = [i32]
        L.mgrit_q8_blocks.restype = i64
        L.mgrit_q8_pack.argtypes = [i64, i32, C.c_int, vp, i64, vp, vp, vp]
        L.mgrit_q8_pack.restype = C.c_int
        L.mgrit_q8_unpack.argtypes = [i64, i32, C.c_int, vp, vp, vp, i64, vp]
        L.mgrit_q8_unpack.restype = C.c_int
        L.mgrit_layer_norm_forward.argtypes = [nd, vp, i64, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp]
        L.mgrit_layer_norm_forward.restype = C.c_int
        L.mgrit_layer_norm_backward_workspace_bytes.argtypes = [nd]
        L.mgrit_layer_norm_backward_workspace_bytes.restype = C.c_size_t
        L.mgrit_layer_norm_backward.argtypes = [nd, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp,
                                                C.c_size_t, vp]
        L.mgrit_layer_norm_backward.restype = C.c_int
        L.mgrit_q8_weight_grad_workspace_bytes.argtypes = [i64, i32, i32, C.c_int]
        L.mgrit_q8_weight_grad_workspace_bytes.restype = C.c_size_t
        L.mgrit_q8_weight_grad.argtypes = [i64, i32, i32, C.c_int, vp, i64, vp, vp, C.c_float, vp, vp, vp, C.c_size_t,
                                           vp]
        L.mgrit_q8_weight_grad.restype = C.c_int
        L.layer_step_batched.argtypes = [C.POINTER(ModelDesc), C.c_int, C.c_int, vpp, vpp, vpp, vpp, vpp, vp,
                                         C.c_float, vp, C.c_size_t, vp]
        L.layer_step_batched.restype = C.c_int
        L.mgrit_layer_step_static_bytes.argtypes = [C.POINTER(ModelDesc), C.c_int, C.c_int]
        L.mgrit_layer_step_static_bytes.restype = C.c_size_t
        L.layer_step_batched_static.argtypes = [C.POINTER(ModelDesc), C.c_int, C.c_int, vpp, vpp, vpp, vpp, vpp, vp,
                                                C.c_float, vp]
        L.layer_step_batched_static.restype = C.c_int
        L.mgrit_buffered_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.POINTER(BufferOpts),
                                                     C.c_int]
        L.mgrit_buffered_workspace_bytes.restype = C.c_size_t
        L.mgrit_forward_buffered.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.POINTER(BufferOpts), vp, vpp,
                                             vp, vp, vp, vp, C.c_size_t, vp]
        L.mgrit_forward_buffered.restype = C.c_int
        L.mgrit_adjoint_buffered.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.POINTER(BufferOpts), vp, vpp,
                                             vp, vp, vp, vp, vpp, vp, vp, C.c_size_t, vp]
        L.mgrit_adjoint_buffered.restype = C.c_int
        L.mgrit_buffered_linearised_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts),
                                                                C.POINTER(BufferOpts), C.c_int]
        L.mgrit_buffered_linearised_workspace_bytes.restype = C.c_size_t
        L.mgrit_forward_buffered_linearising.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.POINTER(BufferOpts),
                                                         vp, vpp, vp, vp, vp, vp, C.c_size_t, vp, C.c_size_t, C.c_int,
                                                         vp]
        L.mgrit_forward_buffered_linearising.restype = C.c_int
        L.mgrit_adjoint_buffered_linearised.argtypes = L.mgrit_adjoint_buffered.argtypes
        L.mgrit_adjoint_buffered_linearised.restype = C.c_int
        L.mgrit_stacked_workspace_bytes.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.c_int, C.c_int]
        L.mgrit_stacked_workspace_bytes.restype = C.c_size_t
        L.mgrit_forward_stacked.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.c_int, vp, vpp, vp, vp, vp,
                                            C.c_size_t, vp]
        L.mgrit_forward_stacked.restype = C.c_int
        L.mgrit_adjoint_stacked.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.c_int, vp, vpp, vp, vp, vpp, vp,
                                            vp, C.c_size_t, vp]
        L.mgrit_adjoint_stacked.restype = C.c_int
        L.mgrit_forward_stacked_linearising.argtypes = [C.POINTER(ModelDesc), C.POINTER(Opts), C.c_int, vp, vpp, vp,
                                                        vp, vp, C.c_size_t, vp, C.c_size_t, C.c_int, vp]
        L.mgrit_forward_stacked_linearising.restype = C.c_int
        L.mgrit_adjoint_stacked_linearised.argtypes = L.mgrit_adjoint_stacked.argtypes
        L.mgrit_adjoint_stacked_linearised.restype = C.c_int
        L.mgrit_indicator_init.argtypes = [C.POINTER(Indicator), C.c_int, C.c_int, C.c_int, C.c_int, C.c_float]
        L.mgrit_indicator_init.restype = C.c_int
        L.mgrit_indicator_begin_batch.argtypes = [C.POINTER(Indicator)]
        L.mgrit_indicator_begin_batch.restype = C.c_int
        L.mgrit_indicator_end_batch.argtypes = [C.POINTER(Indicator), C.POINTER(C.c_float), C.c_int]
        L.mgrit_indicator_end_batch.restype = C.c_int
        L.mgrit_status_string.argtypes = [C.c_int]
        L.mgrit_status_string.restype = C.c_char_p
        L.mgrit_last_hip_error.argtypes = []
        L.mgrit_last_hip_error.restype = C.c_int
        L.mgrit_set_max_groups_per_launch.argtypes = [C.c_int]
        L.mgrit_set_max_groups_per_launch.restype = None
        L.mgrit_default_groups_per_launch.argtypes = [C.POINTER(ModelDesc), C.c_int]
        L.mgrit_default_groups_per_launch.restype = C.c_int
        L.mgrit_debug_pipeline_chunk.argtypes = [C.c_int]
        L.mgrit_debug_pipeline_chunk.restype = None
        L.mgrit_set_lanes.argtypes = [C.c_int]
        L.mgrit_set_lanes.restype = None
        L.mgrit_debug_force_simple_kernels.argtypes = [C.c_int, C.c_int]
        L.mgrit_debug_force_simple_kernels.restype = None
        L.mgrit_debug_gemm_tile_config.argtypes = [C.c_int]
        L.mgrit_debug_gemm_tile_config.restype = None
        L.mgrit_debug_gradient_slices.argtypes = [C.c_int]
        L.mgrit_debug_gradient_slices.restype = None
        L.mgrit_debug_attention_wide_blocks.argtypes = [C.c_int]
        L.mgrit_debug_attention_wide_blocks.restype = None
        L.mgrit_debug_pipeline_coarse_solve.argtypes = [C.c_int]
        L.mgrit_debug_pipeline_coarse_solve.restype = None
        L.mgrit_profile_enable.argtypes = [C.c_int]
        L.mgrit_profile_enable.restype = C.c_int
        L.mgrit_profile_reset.argtypes = []
        L.mgrit_profile_reset.restype = None
        L.mgrit_profile_read.argtypes = [C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                         C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.mgrit_profile_read.restype = C.c_int
        _lib = L
    return _lib


# ------------------------------------------------------------------ descriptors
def model_desc(wl) -> ModelDesc:
    """ModelDesc from any object with the Workload fields."""
    return ModelDesc(wl.arch, wl.d_model, wl.n_heads, wl.d_ff, wl.batch, wl.seq, wl.mem_seq, wl.dtype,
                     wl.ln_eps)


def mgrit_opts(N, h, cf, levels, iters, relax=1, init_guess=0) -> Opts:
    return Opts(N, h, cf, levels, iters, relax, init_guess)


def mgrit_theta_layout(desc: ModelDesc) -> ThetaLayout:
    out = ThetaLayout()
    st = lib().mgrit_theta_layout(C.byref(desc), C.byref(out))
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_theta_layout")
    return out


def mgrit_workspace_bytes(desc: ModelDesc, opts: Opts, adjoint) -> int:
    """adjoint: 0/False forward, 1/True adjoint, 2 adjoint with parameter gradients."""
    return int(lib().mgrit_workspace_bytes(C.byref(desc), C.byref(opts), int(adjoint)))


def mgrit_linearising_workspace_bytes(desc: ModelDesc, opts: Opts) -> int:
    """Workspace of mgrit_forward with an adjoint_workspace."""
    return int(lib().mgrit_linearising_workspace_bytes(C.byref(desc), C.byref(opts)))


def mgrit_adjoint_q8_workspace_bytes(desc: ModelDesc, opts: Opts, adjoint) -> int:
    """Workspace of mgrit_adjoint on Q8Rows (adjoint: 1, or 2 with parameter gradients)."""
    return int(lib().mgrit_adjoint_q8_workspace_bytes(C.byref(desc), C.byref(opts), int(adjoint)))


def grad_layout(desc: ModelDesc) -> ThetaLayout:
    """Layout of a gradient block: the fp32 parameter block of the same model."""
    d32 = ModelDesc.from_buffer_copy(desc)
    d32.dtype = 0
    return mgrit_theta_layout(d32)


def unpack_grad(desc: ModelDesc, block: torch.Tensor) -> Dict[str, np.ndarray]:
    """Copies a gradient block (uint8 device tensor) back into named float32 arrays."""
    lay = grad_layout(desc)
    raw = block.cpu().numpy()
    out = {}
    for i, name in enumerate(P_NAMES):
        if lay.offset[i] < 0:
            continue
        n = lay.rows[i] * lay.cols[i]
        a = raw[lay.offset[i]:lay.offset[i] + 4 * n].view(np.float32)
        out[name] = a.reshape(lay.rows[i], lay.cols[i]) if lay.cols[i] > 1 else a.copy()
    return out


def mgrit_layer_step_workspace_bytes(desc: ModelDesc, adjoint: bool, n_groups: int) -> int:
    return int(lib().mgrit_layer_step_workspace_bytes(C.byref(desc), int(adjoint), n_groups))


def mgrit_step_evaluations(opts: Opts) -> int:
    return int(lib().mgrit_step_evaluations(C.byref(opts)))


def mgrit_step_depth(opts: Opts) -> int:
    return int(lib().mgrit_step_depth(C.byref(opts)))


def mgrit_indicator_init(iters: int, probe_every: int, mitigation: int = MITIGATE_SERIAL, max_iters: int = 0,
                         threshold: float = 1.0) -> Indicator:
    ind = Indicator()
    st = lib().mgrit_indicator_init(C.byref(ind), iters, probe_every, mitigation, max_iters, threshold)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_indicator_init")
    return ind


def mgrit_indicator_begin_batch(ind: Indicator) -> int:
    return int(lib().mgrit_indicator_begin_batch(C.byref(ind)))


def mgrit_indicator_end_batch(ind: Indicator, resnorm) -> int:
    r = np.ascontiguousarray(resnorm, dtype=np.float32)
    return int(lib().mgrit_indicator_end_batch(C.byref(ind), r.ctypes.data_as(C.POINTER(C.c_float)), r.size))


def mgrit_set_max_groups_per_launch(n: int) -> None:
    lib().mgrit_set_max_groups_per_launch(int(n))


def mgrit_set_lanes(n: int) -> None:
    lib().mgrit_set_lanes(int(n))


def mgrit_set_adjoint_cache(on: bool) -> None:
    """False: no N-layer linearisation cache in the adjoint workspace (recomputed per launch chunk)."""
    lib().mgrit_set_adjoint_cache(int(bool(on)))


PROFILE_CLASSES = {0: "gemm_generic", 1: "attn_fwd", 2: "attn_bwd", 3: "ln_fwd", 4: "ln_vjp", 5: "elementwise",
                   6: "ln_fwd_single", 7: "ln_vjp_single",
                   8: "gemm_mfma_store", 9: "gemm_mfma_gelu", 10: "gemm_mfma_sublayer_sum",
                   11: "gemm_mfma_euler", 12: "gemm_mfma_dgelu", 13: "gemm_mfma_store_f32",
                   14: "gemm_mfma_gelu_prime", 15: "gemm_mfma_gelu_both"}
# the same epilogues launched over a single group (the serial coarse chain)
PROFILE_CLASSES.update({c + 8: n.replace("gemm_mfma_", "gemm_mfma_single_") for c, n in list(PROFILE_CLASSES.items())
                        if c >= 8})
PROFILE_CLASSES[24] = "chain"
PROFILE_CLASSES.update({25: "q8", 26: "norm_fwd", 27: "norm_bwd", 28: "q8_weight_grad"})


def mgrit_profile_enable(max_records: int) -> None:
    st = lib().mgrit_profile_enable(int(max_records))
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_profile_enable")


def mgrit_profile_reset() -> None:
    lib().mgrit_profile_reset()


def mgrit_profile_read() -> Dict[str, dict]:
    """Totals per kernel class since the last reset (synchronise the stream first)."""
    out = {}
    for cls, name in PROFILE_CLASSES.items():
        ms, fl, by, n = C.c_double(), C.c_double(), C.c_double(), C.c_int64()
        st = lib().mgrit_profile_read(cls, C.byref(ms), C.byref(fl), C.byref(by), C.byref(n))
        if st not in (0, -3):
            raise MgritError(st, "mgrit_profile_read")
        if n.value:
            out[name] = {"ms": ms.value, "flops": fl.value, "bytes": by.value, "launches": n.value,
                         "overflow": st == -3}
    return out


def mgrit_measure_mfma_ceiling(scratch: torch.Tensor, iters: int = 20000, stream=None) -> float:
    """TFLOP/s of the register-resident MFMA loop (scratch: device tensor of at least 512 KiB)."""
    out = C.c_double()
    st = lib().mgrit_measure_mfma_ceiling(scratch.data_ptr(), scratch.numel() * scratch.element_size(), int(iters),
                                          C.byref(out), _stream_handle(stream))
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_measure_mfma_ceiling")
    return out.value


def mgrit_measure_copy_ceiling(src: torch.Tensor, dst: torch.Tensor, stream=None) -> float:
    """GB/s (read + written) of a grid-stride copy of src into dst (device tensors of equal size)."""
    out = C.c_double()
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    st = lib().mgrit_measure_copy_ceiling(src.data_ptr(), dst.data_ptr(), nbytes, C.byref(out), _stream_handle(stream))
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_measure_copy_ceiling")
    return out.value


def mgrit_measure_event_bracket(stream=None) -> float:
    """Microseconds that an event pair adds to the launch it brackets (median around an empty kernel)."""
    out = C.c_double()
    st = lib().mgrit_measure_event_bracket(C.byref(out), _stream_handle(stream))
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_measure_event_bracket")
    return out.value


# ------------------------------------------------------------------ parameter packing (byte copies only)
def pack_theta(desc: ModelDesc, params: Dict[str, np.ndarray], device="cuda") -> torch.Tensor:
    """One layer's named fp32 arrays -> packed device block (uint8 tensor) in the library's layout."""
    lay = mgrit_theta_layout(desc)
    host = torch.zeros(int(lay.block_bytes), dtype=torch.uint8)
    for i, name in enumerate(P_NAMES):
        off = int(lay.offset[i])
        if off < 0:
            continue
        a = torch.from_numpy(np.ascontiguousarray(params[name], dtype=np.float32))
        assert a.numel() == lay.rows[i] * lay.cols[i], name
        if lay.elem_bytes[i] == 2:
            raw = a.to(torch.bfloat16).view(torch.uint8).reshape(-1)
        else:
            raw = a.view(torch.uint8).reshape(-1)
        host[off:off + raw.numel()] = raw
    return host.to(device)


def _ptr(t: Optional[torch.Tensor]) -> C.c_void_p:
    return C.c_void_p(0 if t is None else t.data_ptr())


def _ptr_array(ts: Optional[Sequence[torch.Tensor]]):
    if ts is None:
        return None
    arr = (C.c_void_p * len(ts))(*[t.data_ptr() for t in ts])
    return arr


def _stream_handle(stream: Optional[torch.cuda.Stream]) -> C.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _check_state(t: torch.Tensor, shape, name: str):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a tensor, got {type(t).__name__}")
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and tuple(t.shape) == tuple(shape)):
        raise ValueError(f"{name}: expected contiguous fp32 device tensor of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


# ------------------------------------------------------------------ entry points
def mgrit_forward(desc: ModelDesc, opts: Opts, Z0: torch.Tensor, theta: List[torch.Tensor],
                  memory: Optional[torch.Tensor] = None, Z_all: Optional[torch.Tensor] = None,
                  resnorm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None, adjoint_workspace: Optional[torch.Tensor] = None,
                  with_gradients: bool = False):
    """Returns (Z_all [(N+1),T,d], resnorm [iters]).  Buffers are allocated here if not given.
    adjoint_workspace: call mgrit_forward_linearising instead, which also leaves the internals of its
    closing relaxation there for mgrit_adjoint(..., workspace=adjoint_workspace, linearised=True)."""
    T, d = desc.batch * desc.seq, desc.d_model
    _check_state(Z0, (T, d), "Z0")
    if len(theta) != opts.N:
        raise ValueError("theta must hold N blocks")
    handle, other = _on(stream, Z0.get_device())
    if Z_all is None:
        Z_all = _new((opts.N + 1, T, d), torch.float32, Z0.device, other)
    _check_state(Z_all, (opts.N + 1, T, d), "Z_all")
    if resnorm is None:
        resnorm = _new_zeros(max(opts.iters, 1), Z0.device, other)
    if workspace is None:
        need = (mgrit_workspace_bytes(desc, opts, False) if adjoint_workspace is None else
                mgrit_linearising_workspace_bytes(desc, opts))
        workspace = _new((max(need, 256),), torch.uint8, Z0.device, other)
    if adjoint_workspace is not None:
        st = lib().mgrit_forward_linearising(C.byref(desc), C.byref(opts), _ptr(Z0), _ptr_array(theta), _ptr(memory),
                                             _ptr(Z_all), _ptr(resnorm), _ptr(workspace), workspace.numel(),
                                             _ptr(adjoint_workspace), adjoint_workspace.numel(),
                                             int(bool(with_gradients)), handle)
        if st != MGRIT_OK:
            raise MgritError(st, "mgrit_forward_linearising")
    else:
        st = lib().mgrit_forward(C.byref(desc), C.byref(opts), _ptr(Z0), _ptr_array(theta), _ptr(memory),
                                 _ptr(Z_all), _ptr(resnorm), _ptr(workspace), workspace.numel(), handle)
        if st != MGRIT_OK:
            raise MgritError(st, "mgrit_forward")
    if other is not None:
        _in_use(other, Z0, *theta, memory, Z_all, resnorm, workspace, adjoint_workspace)
    return Z_all, resnorm


def mgrit_adjoint(desc: ModelDesc, opts: Opts, Z_all, theta: List[torch.Tensor],
                  lambda_N: torch.Tensor, memory: Optional[torch.Tensor] = None,
                  lambda_all: Optional[torch.Tensor] = None, resnorm: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                  dtheta: Optional[List[torch.Tensor]] = None, dmemory: Optional[torch.Tensor] = None,
                  linearised: bool = False):
    """Returns (lambda_all [(N+1),T,d], resnorm [iters]).  dtheta: N uint8 device tensors of
    grad_layout(desc).block_bytes each, filled with the parameter gradients; dmemory: fp32
    [batch*mem_seq, d] device tensor filled with the gradient of the cross-attention memory.
    linearised: call mgrit_adjoint_linearised (workspace = the adjoint_workspace that mgrit_forward filled).
    Z_all may be Q8Rows of that shape, mgrit_q8_pack(Z_all): mgrit_adjoint_q8 (workspace:
    mgrit_adjoint_q8_workspace_bytes).
    stream: where the call is enqueued, behind what the caller has put before it there; what is allocated here belongs to it."""
    if linearised and workspace is None:
        raise ValueError("linearised: pass the adjoint workspace that the forward call filled")
    T, d = desc.batch * desc.seq, desc.d_model
    q8 = isinstance(Z_all, Q8Rows)
    if q8:
        if linearised:
            raise ValueError("linearised: the adjoint of that pair takes Z_all as the forward call left it")
        if Z_all.shape != (opts.N + 1, T, d):
            raise ValueError(f"Z_all: expected 8-bit rows of shape {(opts.N + 1, T, d)}, got {tuple(Z_all.shape)}")
        _check_q8(Z_all, "Z_all", _device_of(Z_all.q, "Z_all"))
    else:
        _check_state(Z_all, (opts.N + 1, T, d), "Z_all")
    _check_state(lambda_N, (T, d), "lambda_N")
    if len(theta) != opts.N:
        raise ValueError("theta must hold N blocks")
    handle, other = _on(stream, lambda_N.get_device())
    if lambda_all is None:
        lambda_all = _new((opts.N + 1, T, d), torch.float32, Z_all.device, other)
    _check_state(lambda_all, (opts.N + 1, T, d), "lambda_all")
    if resnorm is None:
        resnorm = _new_zeros(max(opts.iters, 1), Z_all.device, other)
    if dtheta is not None and len(dtheta) != opts.N:
        raise ValueError("dtheta must hold N blocks")
    if dmemory is not None:
        _check_state(dmemory, (desc.batch * desc.mem_seq, d), "dmemory")
    query = mgrit_adjoint_q8_workspace_bytes if q8 else mgrit_workspace_bytes
    need = query(desc, opts, 2 if (dtheta is not None or dmemory is not None) else 1)
    if workspace is None:
        workspace = _new((max(need, 256),), torch.uint8, Z_all.device, other)
    name = "mgrit_adjoint_q8" if q8 else "mgrit_adjoint_linearised" if linearised else "mgrit_adjoint"
    states = (_ptr(Z_all.q), _ptr(Z_all.scale)) if q8 else (_ptr(Z_all),)
    st = getattr(lib(), name)(C.byref(desc), C.byref(opts), *states, _ptr_array(theta), _ptr(memory),
                              _ptr(lambda_N), _ptr(lambda_all), _ptr(dmemory), _ptr_array(dtheta), _ptr(resnorm),
                              _ptr(workspace), workspace.numel(), handle)
    if st != MGRIT_OK:
        raise MgritError(st, name)
    if other is not None:
        _in_use(other, Z_all, *theta, memory, lambda_N, lambda_all, dmemory, *(dtheta or ()), resnorm, workspace)
    return lambda_all, resnorm


def layer_step_batched(desc: ModelDesc, adjoint: bool, inputs: List[torch.Tensor], outputs: List[torch.Tensor],
                       theta: List[torch.Tensor], hstep: float,
                       lin_state: Optional[List[torch.Tensor]] = None,
                       rhs: Optional[List[torch.Tensor]] = None, memory: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """out[g] = in[g] + hstep*F(in[g]; theta[g]) (+rhs[g]), or its adjoint at lin_state[g]."""
    G = len(inputs)
    T, d = desc.batch * desc.seq, desc.d_model
    for t in list(inputs) + list(outputs) + list(lin_state or []) + list(rhs or []):
        _check_state(t, (T, d), "state")
    handle, other = _on(stream, inputs[0].get_device() if inputs else torch.cuda.current_device())
    need = mgrit_layer_step_workspace_bytes(desc, adjoint, G)
    if workspace is None:
        workspace = _new((max(need, 256),), torch.uint8, inputs[0].device, other)
    st = lib().layer_step_batched(C.byref(desc), int(adjoint), G, _ptr_array(inputs), _ptr_array(outputs),
                                  _ptr_array(theta), _ptr_array(lin_state), _ptr_array(rhs), _ptr(memory),
                                  float(hstep), _ptr(workspace), workspace.numel(), handle)
    if st != MGRIT_OK:
        raise MgritError(st, "layer_step_batched")
    if other is not None:
        _in_use(other, *inputs, *outputs, *theta, *(lin_state or ()), *(rhs or ()), memory, workspace)
    return outputs


STATIC_SCRATCH_BYTES = 256 << 20     # MGRIT_STATIC_SCRATCH_BYTES of the header


def mgrit_layer_step_static_bytes(desc: ModelDesc, adjoint: bool, n_groups: int) -> int:
    return int(lib().mgrit_layer_step_static_bytes(C.byref(desc), int(adjoint), n_groups))


def layer_step_batched_static(desc: ModelDesc, adjoint: bool, inputs: List[torch.Tensor],
                              outputs: List[torch.Tensor], theta: List[torch.Tensor], hstep: float,
                              lin_state: Optional[List[torch.Tensor]] = None,
                              rhs: Optional[List[torch.Tensor]] = None, memory: Optional[torch.Tensor] = None,
                              stream: Optional[torch.cuda.Stream] = None):
    """layer_step_batched on the library's own fixed scratch array: no workspace, nothing allocated."""
    G = len(inputs)
    T, d = desc.batch * desc.seq, desc.d_model
    for t in list(inputs) + list(outputs) + list(lin_state or []) + list(rhs or []):
        _check_state(t, (T, d), "state")
    handle, other = _on(stream, inputs[0].get_device() if inputs else torch.cuda.current_device())
    st = lib().layer_step_batched_static(C.byref(desc), int(adjoint), G, _ptr_array(inputs), _ptr_array(outputs),
                                         _ptr_array(theta), _ptr_array(lin_state), _ptr_array(rhs), _ptr(memory),
                                         float(hstep), handle)
    if st != MGRIT_OK:
        raise MgritError(st, "layer_step_batched_static")
    if other is not None:
        _in_use(other, *inputs, *outputs, *theta, *(lin_state or ()), *(rhs or ()), memory)
    return outputs


def mgrit_buffered_workspace_bytes(desc: ModelDesc, opts: Opts, buf: BufferOpts, adjoint) -> int:
    return int(lib().mgrit_buffered_workspace_bytes(C.byref(desc), C.byref(opts), C.byref(buf), int(adjoint)))


def mgrit_buffered_linearised_workspace_bytes(desc: ModelDesc, opts: Opts, buf: BufferOpts, with_gradients) -> int:
    return int(lib().mgrit_buffered_linearised_workspace_bytes(C.byref(desc), C.byref(opts), C.byref(buf),
                                                               int(bool(with_gradients))))


def mgrit_forward_buffered(desc: ModelDesc, opts: Opts, buf: BufferOpts, Z0: torch.Tensor,
                           theta: List[torch.Tensor], memory: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None,
                           adjoint_workspace: Optional[torch.Tensor] = None, with_gradients: bool = False):
    """Serial open / close layers around the MGRIT middle.  Returns (Z_all, resnorm).
    adjoint_workspace (mgrit_buffered_linearised_workspace_bytes): mgrit_forward_buffered_linearising."""
    T, d = desc.batch * desc.seq, desc.d_model
    n = buf.n_open + opts.N + buf.n_close
    _check_state(Z0, (T, d), "Z0")
    if len(theta) != n:
        raise ValueError("theta must hold n_open + N + n_close blocks")
    handle, other = _on(stream, Z0.get_device())
    Z_all = _new((n + 1, T, d), torch.float32, Z0.device, other)
    resnorm = _new_zeros(max(opts.iters, 1), Z0.device, other)
    ws = _new((max(mgrit_buffered_workspace_bytes(desc, opts, buf, 0), 256),), torch.uint8, Z0.device, other)
    if adjoint_workspace is not None:
        st = lib().mgrit_forward_buffered_linearising(C.byref(desc), C.byref(opts), C.byref(buf), _ptr(Z0),
                                                      _ptr_array(theta), _ptr(memory), _ptr(Z_all), _ptr(resnorm),
                                                      _ptr(ws), ws.numel(), _ptr(adjoint_workspace),
                                                      adjoint_workspace.numel(), int(bool(with_gradients)),
                                                      handle)
        if st != MGRIT_OK:
            raise MgritError(st, "mgrit_forward_buffered_linearising")
    else:
        st = lib().mgrit_forward_buffered(C.byref(desc), C.byref(opts), C.byref(buf), _ptr(Z0), _ptr_array(theta),
                                          _ptr(memory), _ptr(Z_all), _ptr(resnorm), _ptr(ws), ws.numel(), handle)
        if st != MGRIT_OK:
            raise MgritError(st, "mgrit_forward_buffered")
    if other is not None:
        _in_use(other, Z0, *theta, memory, Z_all, resnorm, ws, adjoint_workspace)
    return Z_all, resnorm


def mgrit_adjoint_buffered(desc: ModelDesc, opts: Opts, buf: BufferOpts, Z_all: torch.Tensor,
                           theta: List[torch.Tensor], lambda_N: torch.Tensor, memory: Optional[torch.Tensor] = None,
                           dtheta: Optional[List[torch.Tensor]] = None,
                           stream: Optional[torch.cuda.Stream] = None, workspace: Optional[torch.Tensor] = None,
                           linearised: bool = False):
    """Returns (lambda_all, resnorm) of the buffered network; dtheta as in mgrit_adjoint.
    linearised: mgrit_adjoint_buffered_linearised on the workspace the forward call filled."""
    if linearised and workspace is None:
        raise ValueError("linearised: pass the adjoint workspace that the forward call filled")
    T, d = desc.batch * desc.seq, desc.d_model
    n = buf.n_open + opts.N + buf.n_close
    _check_state(Z_all, (n + 1, T, d), "Z_all")
    _check_state(lambda_N, (T, d), "lambda_N")
    if len(theta) != n or (dtheta is not None and len(dtheta) != n):
        raise ValueError("theta / dtheta must hold n_open + N + n_close blocks")
    handle, other = _on(stream, Z_all.get_device())
    lambda_all = _new(Z_all.shape, torch.float32, Z_all.device, other)
    resnorm = _new_zeros(max(opts.iters, 1), Z_all.device, other)
    need = mgrit_buffered_workspace_bytes(desc, opts, buf, 2 if dtheta is not None else 1)
    ws = workspace if workspace is not None else _new((max(need, 256),), torch.uint8, Z_all.device, other)
    entry = lib().mgrit_adjoint_buffered_linearised if linearised else lib().mgrit_adjoint_buffered
    st = entry(C.byref(desc), C.byref(opts), C.byref(buf), _ptr(Z_all), _ptr_array(theta),
               _ptr(memory), _ptr(lambda_N), _ptr(lambda_all), None, _ptr_array(dtheta),
               _ptr(resnorm), _ptr(ws), ws.numel(), handle)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_adjoint_buffered_linearised" if linearised else "mgrit_adjoint_buffered")
    if other is not None:
        _in_use(other, Z_all, *theta, memory, lambda_N, lambda_all, *(dtheta or ()), resnorm, ws)
    return lambda_all, resnorm


# ---- stacked encoder-decoder grid -------------------------------------------------------------
def encoder_desc(desc: ModelDesc) -> ModelDesc:
    """The encoder half of a stacked grid described by its decoder `desc`."""
    return ModelDesc(0, desc.d_model, desc.n_heads, desc.d_ff, desc.batch, desc.mem_seq, 0, desc.dtype, desc.ln_eps)


def mgrit_stacked_workspace_bytes(desc: ModelDesc, opts: Opts, n_enc: int, adjoint: int) -> int:
    return int(lib().mgrit_stacked_workspace_bytes(C.byref(desc), C.byref(opts), int(n_enc), int(adjoint)))


def mgrit_forward_stacked(desc: ModelDesc, opts: Opts, n_enc: int, Z0: torch.Tensor, theta: List[torch.Tensor],
                          Z_all: Optional[torch.Tensor] = None, resnorm: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                          adjoint_workspace: Optional[torch.Tensor] = None, with_gradients: bool = False):
    """One MGRIT grid over n_enc encoder layers followed by decoder layers; state rows = encoder
    tokens then decoder tokens.  Returns (Z_all, resnorm).  Buffers are allocated here if not given.
    adjoint_workspace: mgrit_forward_stacked_linearising (see mgrit_forward)."""
    T, d = desc.batch * (desc.mem_seq + desc.seq), desc.d_model
    _check_state(Z0, (T, d), "Z0")
    if len(theta) != opts.N:
        raise ValueError("theta must hold N blocks")
    handle, other = _on(stream, Z0.get_device())
    if Z_all is None:
        Z_all = _new((opts.N + 1, T, d), torch.float32, Z0.device, other)
    _check_state(Z_all, (opts.N + 1, T, d), "Z_all")
    if resnorm is None:
        resnorm = _new_zeros(max(opts.iters, 1), Z0.device, other)
    if workspace is None:
        need = mgrit_stacked_workspace_bytes(desc, opts, n_enc, 0)
        workspace = _new((max(need, 256),), torch.uint8, Z0.device, other)
    if adjoint_workspace is not None:
        st = lib().mgrit_forward_stacked_linearising(C.byref(desc), C.byref(opts), int(n_enc), _ptr(Z0),
                                                     _ptr_array(theta), _ptr(Z_all), _ptr(resnorm), _ptr(workspace),
                                                     workspace.numel(), _ptr(adjoint_workspace),
                                                     adjoint_workspace.numel(), int(bool(with_gradients)),
                                                     handle)
        if st != MGRIT_OK:
            raise MgritError(st, "mgrit_forward_stacked_linearising")
    else:
        st = lib().mgrit_forward_stacked(C.byref(desc), C.byref(opts), int(n_enc), _ptr(Z0), _ptr_array(theta),
                                         _ptr(Z_all), _ptr(resnorm), _ptr(workspace), workspace.numel(), handle)
        if st != MGRIT_OK:
            raise MgritError(st, "mgrit_forward_stacked")
    if other is not None:
        _in_use(other, Z0, *theta, Z_all, resnorm, workspace, adjoint_workspace)
    return Z_all, resnorm


def mgrit_adjoint_stacked(desc: ModelDesc, opts: Opts, n_enc: int, Z_all: torch.Tensor, theta: List[torch.Tensor],
                          lambda_N: torch.Tensor, dtheta: Optional[List[torch.Tensor]] = None,
                          lambda_all: Optional[torch.Tensor] = None, resnorm: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                          linearised: bool = False):
    """Returns (lambda_all, resnorm) of the stacked grid; dtheta as in mgrit_adjoint (encoder
    layers' blocks in the encoder's fp32 layout, decoder layers' in the decoder's).
    linearised: mgrit_adjoint_stacked_linearised on the workspace the forward call filled."""
    if linearised and workspace is None:
        raise ValueError("linearised: pass the adjoint workspace that the forward call filled")
    T, d = desc.batch * (desc.mem_seq + desc.seq), desc.d_model
    _check_state(Z_all, (opts.N + 1, T, d), "Z_all")
    _check_state(lambda_N, (T, d), "lambda_N")
    if len(theta) != opts.N or (dtheta is not None and len(dtheta) != opts.N):
        raise ValueError("theta / dtheta must hold N blocks")
    handle, other = _on(stream, Z_all.get_device())
    if lambda_all is None:
        lambda_all = _new(Z_all.shape, torch.float32, Z_all.device, other)
    _check_state(lambda_all, (opts.N + 1, T, d), "lambda_all")
    if resnorm is None:
        resnorm = _new_zeros(max(opts.iters, 1), Z_all.device, other)
    if workspace is None:
        need = mgrit_stacked_workspace_bytes(desc, opts, n_enc, 2 if dtheta is not None else 1)
        workspace = _new((max(need, 256),), torch.uint8, Z_all.device, other)
    entry = lib().mgrit_adjoint_stacked_linearised if linearised else lib().mgrit_adjoint_stacked
    st = entry(C.byref(desc), C.byref(opts), int(n_enc), _ptr(Z_all), _ptr_array(theta),
               _ptr(lambda_N), _ptr(lambda_all), _ptr_array(dtheta), _ptr(resnorm),
               _ptr(workspace), workspace.numel(), handle)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_adjoint_stacked_linearised" if linearised else "mgrit_adjoint_stacked")
    if other is not None:
        _in_use(other, Z_all, *theta, lambda_N, lambda_all, *(dtheta or ()), resnorm, workspace)
    return lambda_all, resnorm


# ---- operators around the solves: 8-bit rows, LayerNorm of rows, gradients from 8-bit rows ------------
# Like the solves, the operators are outside autograd: what they return has no graph behind it, also where an operand requires a
# gradient.  A program calls the backward pass itself (or wraps both in a torch.autograd.Function).
# (Small calls take as long as the host needs for them: what is asked of tensors below is what costs least.)
Q8_BLOCK = 32                        # MGRIT_Q8_BLOCK of the header
MOST_COLS = 2 ** 31 - 1              # a row's length has 32 bits in the header, and ctypes cuts what has more
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class Q8Rows:
    """Rows kept in 8 bits: q, int8 [..., 32 * blocks], and scale, uint8 [..., blocks], standing for rows of `cols`
    elements.  rows[i] is a view of the rows under a leading index (or slice)."""
    __slots__ = ("q", "scale", "cols")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, cols: int):
        blocks = (cols + Q8_BLOCK - 1) // Q8_BLOCK
        at, kept = scale.shape, q.shape
        if (not 0 < cols <= MOST_COLS or q.dtype is not torch.int8 or scale.dtype is not torch.uint8 or len(at) < 1 or len(kept) != len(at)
                or at[-1] != blocks or kept[-1] != blocks * Q8_BLOCK or kept[:-1] != at[:-1]):
            raise ValueError(f"8-bit rows of {cols} elements: expected int8 [..., {blocks * Q8_BLOCK}] and uint8 [..., "
                             f"{blocks}], got {q.dtype} {tuple(q.shape)} and {scale.dtype} {tuple(scale.shape)}")
        self.q, self.scale, self.cols = q, scale, int(cols)

    @classmethod
    def _of(cls, q: torch.Tensor, scale: torch.Tensor, cols: int) -> "Q8Rows":
        """Without the checks, for tensors made here."""
        rows = object.__new__(cls)
        rows.q, rows.scale, rows.cols = q, scale, cols
        return rows

    @property
    def shape(self) -> torch.Size:
        return torch.Size((*self.q.shape[:-1], self.cols))

    @property
    def device(self) -> torch.device:
        return self.q.device

    @property
    def rows(self) -> int:
        return self.scale.numel() // self.scale.shape[-1]

    def __getitem__(self, index) -> "Q8Rows":
        if self.q.dim() < 2 or not isinstance(index, (int, slice)):
            raise IndexError("8-bit rows take one leading index or slice")
        return Q8Rows(self.q[index], self.scale[index], self.cols)


def q8_empty(shape, device="cuda") -> Q8Rows:
    """Uninitialised 8-bit rows for a tensor of that shape."""
    *lead, cols = shape
    if not 0 < cols <= MOST_COLS:
        raise ValueError(f"8-bit rows: expected rows of 1 to 2^31 - 1 elements, got {tuple(shape)}")
    blocks = (cols + Q8_BLOCK - 1) // Q8_BLOCK
    return Q8Rows._of(torch.empty(*lead, blocks * Q8_BLOCK, dtype=torch.int8, device=device),
                      torch.empty(*lead, blocks, dtype=torch.uint8, device=device), cols)


def _device_of(t: torch.Tensor, name: str) -> int:
    """Index of a call's device: that of its first operand, which has to be the current one."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a tensor, got {type(t).__name__}")
    device = t.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: expected a tensor on the current device, got one on {t.device}")
    return device


def _check_device(t: torch.Tensor, name: str, device: int):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a tensor, got {type(t).__name__}")
    if t.get_device() != device:
        raise ValueError(f"{name}: expected a tensor on the current device, got one on {t.device}")


def _is_q8(r: Q8Rows, name: str) -> Q8Rows:
    if not isinstance(r, Q8Rows):
        raise ValueError(f"{name}: expected Q8Rows, got {type(r).__name__}")
    return r


def _check_q8(r: Q8Rows, name: str, device: int, shape=None):
    q, scale = _is_q8(r, name).q, r.scale
    if q.get_device() != device or scale.get_device() != device:
        raise ValueError(f"{name}: expected tensors on the current device, got some on {q.device} and {scale.device}")
    if not (q.is_contiguous() and scale.is_contiguous()):
        raise ValueError(f"{name}: expected contiguous 8-bit rows")
    if shape is not None and (r.cols != shape[-1] or q.shape[:-1] != shape[:-1]):
        raise ValueError(f"{name}: expected 8-bit rows of shape {tuple(shape)}, got {tuple(r.shape)}")


def _check_rows(t: torch.Tensor, name: str, device: int, shape=None):
    """(rows, cols, stride) of a matrix argument: leading dimensions that lie one behind the other are rows."""
    _check_device(t, name, device)
    own = t.shape
    if t.dtype not in _DTYPES or len(own) < 1 or not 0 < own[-1] <= MOST_COLS or (shape is not None and own != shape):
        raise ValueError(f"{name}: expected fp32 or bf16 rows of at most 2^31 - 1 elements" + (f" of shape {tuple(shape)}" if shape is not None else "") +
                         f", got {t.dtype} {tuple(own)}")
    cols = own[-1]
    if t.is_contiguous():
        return t.numel() // cols, cols, cols
    if len(own) == 2 and t.stride(1) == 1 and (own[0] == 1 or t.stride(0) >= cols):
        return own[0], cols, max(t.stride(0), cols)
    raise ValueError(f"{name}: expected contiguous rows, or a matrix of rows at one distance, got strides {t.stride()}")


def _check_vector(t: Optional[torch.Tensor], n: int, name: str, device: int) -> Optional[int]:
    """Address of a vector argument, None without."""
    if t is None:
        return None
    _check_device(t, name, device)
    if t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous fp32 vector of {n}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _on(stream: Optional[torch.cuda.Stream], device: int):
    """(handle, stream if it is not the current one): where a call is enqueued."""
    current = torch._C._cuda_getCurrentRawStream(device)
    if stream is None:
        return current, None
    if stream.device_index != device:
        raise ValueError(f"stream: expected one of the current device, got one of device {stream.device_index}")
    if stream.cuda_stream == current:
        return current, None
    return stream.cuda_stream, stream


def _new(shape, dtype: torch.dtype, device: torch.device, other: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """A new tensor that belongs to the stream its call is enqueued on."""
    if other is None:
        return torch.empty(*shape, dtype=dtype, device=device)          # (a tuple as it is takes 0.8 us longer)
    with torch.cuda.stream(other):
        return torch.empty(*shape, dtype=dtype, device=device)


def _new_zeros(n: int, device: torch.device, other: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """fp32 zeros, filled on the stream the call is enqueued on."""
    if other is None:
        return torch.zeros(n, dtype=torch.float32, device=device)
    with torch.cuda.stream(other):
        return torch.zeros(n, dtype=torch.float32, device=device)


def _new_q8(shape, device: torch.device, other: Optional[torch.cuda.Stream]) -> Q8Rows:
    if other is None:
        return q8_empty(shape, device)
    with torch.cuda.stream(other):
        return q8_empty(shape, device)


def _in_use(other: torch.cuda.Stream, *operands):
    """After a call on another stream than the current one: the operands' memory is not handed out again before it ran."""
    for t in operands:
        for u in ((t.q, t.scale) if isinstance(t, Q8Rows) else (t,)):
            if u is not None:
                u.record_stream(other)


def _workspace(given: Optional[torch.Tensor], need: int, device: torch.device, other):
    """(tensor, address, bytes): the caller's, or a new one if the call needs any."""
    if given is None:
        given = _new((need,), torch.uint8, device, other) if need else None
        return given, given.data_ptr() if need else None, need
    if given.dtype != torch.uint8 or not given.is_contiguous() or given.device != device:
        raise ValueError("workspace: expected a contiguous uint8 tensor on the operands' device")
    return given, given.data_ptr(), given.numel()


def _vector(given: Optional[torch.Tensor], n: int, name: str, device: int, like: torch.Tensor, other):
    """(tensor, address): the caller's output vector, or a new one."""
    if given is None:
        given = _new((n,), torch.float32, like.device, other)
        return given, given.data_ptr()
    return given, _check_vector(given, n, name, device)


def _c_int32(n: int) -> int:
    if n > MOST_COLS:
        raise ValueError(f"expected a length of at most 2^31 - 1, got {n}")
    return n


def mgrit_q8_blocks(cols: int) -> int:
    return int(lib().mgrit_q8_blocks(_c_int32(int(cols))))


def mgrit_q8_pack(x: torch.Tensor, out: Optional[Q8Rows] = None, stream: Optional[torch.cuda.Stream] = None) -> Q8Rows:
    """The 8-bit rows of x (fp32 or bf16, [..., cols])."""
    device = _device_of(x, "x")
    rows, cols, stride = _check_rows(x, "x", device)
    handle, other = _on(stream, device)
    if out is None:
        out = _new_q8(x.shape, x.device, other)
    else:
        _check_q8(out, "out", device, x.shape)
    st = lib().mgrit_q8_pack(rows, cols, _DTYPES[x.dtype], x.data_ptr(), stride, out.q.data_ptr(), out.scale.data_ptr(), handle)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_q8_pack")
    if other is not None:
        _in_use(other, x, out)
    return out


def mgrit_q8_unpack(x: Q8Rows, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """What 8-bit rows stand for, as fp32 or bf16 (exactly, in either); with out, in its type."""
    device = _device_of(_is_q8(x, "x").q, "x")
    _check_q8(x, "x", device)
    handle, other = _on(stream, device)
    if out is None:
        if dtype not in _DTYPES:
            raise ValueError(f"dtype: expected float32 or bfloat16, got {dtype}")
        out = _new(x.shape, dtype, x.device, other)
        rows, cols = x.rows, x.cols
        stride = cols
    else:
        rows, cols, stride = _check_rows(out, "out", device, x.shape)
    st = lib().mgrit_q8_unpack(rows, cols, _DTYPES[out.dtype], x.q.data_ptr(), x.scale.data_ptr(), out.data_ptr(), stride, handle)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_q8_unpack")
    if other is not None:
        _in_use(other, x, out)
    return out


def mgrit_layer_norm_forward(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                             eps: float = 1e-5, y: Optional[torch.Tensor] = None, y_dtype: Optional[torch.dtype] = None,
                             mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None,
                             x_q8: Optional[Q8Rows] = None, y_q8: Optional[Q8Rows] = None,
                             stream: Optional[torch.cuda.Stream] = None):
    """Returns (y, mean, rstd): LayerNorm of the rows of x (fp32 or bf16, [..., cols]) with y of y_dtype (x's own by
    default) and the rows' statistics, fp32 [rows].  x_q8, y_q8: 8-bit rows (q8_empty) filled from the same pass.
    Not recorded by autograd: gradients come from mgrit_layer_norm_backward."""
    device = _device_of(x, "x")
    rows, cols, ldx = _check_rows(x, "x", device)
    handle, other = _on(stream, device)
    if y is None:
        y_dtype = x.dtype if y_dtype is None else y_dtype
        if y_dtype not in _DTYPES:
            raise ValueError(f"y_dtype: expected float32 or bfloat16, got {y_dtype}")
        y, ldy = _new(x.shape, y_dtype, x.device, other), cols
    else:
        _, _, ldy = _check_rows(y, "y", device, x.shape)
        if y_dtype is not None and y_dtype != y.dtype:
            raise ValueError(f"y: expected {y_dtype}, got {y.dtype}")
    mean, mean_at = _vector(mean, rows, "mean", device, x, other)
    rstd, rstd_at = _vector(rstd, rows, "rstd", device, x, other)
    xq = xs = yq = ys = None
    if x_q8 is not None:
        _check_q8(x_q8, "x_q8", device, x.shape)
        xq, xs = x_q8.q.data_ptr(), x_q8.scale.data_ptr()
    if y_q8 is not None:
        _check_q8(y_q8, "y_q8", device, x.shape)
        yq, ys = y_q8.q.data_ptr(), y_q8.scale.data_ptr()
    desc = NormDesc(rows, cols, _DTYPES[x.dtype], _DTYPES[y.dtype], eps)
    st = lib().mgrit_layer_norm_forward(desc, x.data_ptr(), ldx, _check_vector(gamma, cols, "gamma", device),
                                        _check_vector(beta, cols, "beta", device), y.data_ptr(), ldy,
                                        mean_at, rstd_at, xq, xs, yq, ys, handle)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_layer_norm_forward")
    if other is not None:
        _in_use(other, x, gamma, beta, y, mean, rstd, x_q8, y_q8)
    return y, mean, rstd


def mgrit_layer_norm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().mgrit_layer_norm_backward_workspace_bytes(NormDesc(rows, _c_int32(cols), 0, 0, 1e-5)))


def mgrit_layer_norm_backward(dy: torch.Tensor, x, gamma: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                              dx_dtype: Optional[torch.dtype] = None, dx: Optional[torch.Tensor] = None,
                              dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Returns (dx, dgamma, dbeta) of mgrit_layer_norm_forward for the cotangent dy.  x: its input, or the Q8Rows kept of
    it; mean, rstd: as it returned them.  dx has x's type (8-bit rows: dx_dtype, fp32 by default)."""
    device = _device_of(dy, "dy")
    rows, cols, lddy = _check_rows(dy, "dy", device)
    if isinstance(x, Q8Rows):
        _check_q8(x, "x", device, dy.shape)
        x_at, ldx, xq, xs = None, 0, x.q.data_ptr(), x.scale.data_ptr()
        x_dtype = torch.float32 if dx_dtype is None else dx_dtype
    else:
        _, _, ldx = _check_rows(x, "x", device, dy.shape)
        x_at, xq, xs, x_dtype = x.data_ptr(), None, None, x.dtype
    if x_dtype not in _DTYPES or (dx_dtype is not None and dx_dtype != x_dtype):
        raise ValueError(f"dx_dtype: dx has the type of x, float32 or bfloat16, got {dx_dtype}")
    handle, other = _on(stream, device)
    if dx is None:
        dx, lddx = _new(dy.shape, x_dtype, dy.device, other), cols
    else:
        _, _, lddx = _check_rows(dx, "dx", device, dy.shape)
        if dx.dtype != x_dtype:
            raise ValueError(f"dx: expected {x_dtype}, got {dx.dtype}")
    dgamma, dgamma_at = _vector(dgamma, cols, "dgamma", device, dy, other)
    dbeta, dbeta_at = _vector(dbeta, cols, "dbeta", device, dy, other)
    desc, L = NormDesc(rows, cols, _DTYPES[x_dtype], _DTYPES[dy.dtype], 1e-5), lib()
    ws, ws_at, ws_bytes = _workspace(workspace, L.mgrit_layer_norm_backward_workspace_bytes(desc), dy.device, other)
    st = L.mgrit_layer_norm_backward(desc, dy.data_ptr(), lddy, x_at, ldx, xq, xs, _check_vector(gamma, cols, "gamma", device),
                                     _check_vector(mean, rows, "mean", device), _check_vector(rstd, rows, "rstd", device),
                                     dx.data_ptr(), lddx, dgamma_at, dbeta_at, ws_at, ws_bytes, handle)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_layer_norm_backward")
    if other is not None:
        _in_use(other, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    return dx, dgamma, dbeta


def mgrit_q8_weight_grad_workspace_bytes(rows: int, out_features: int, in_features: int, dtype: torch.dtype) -> int:
    return int(lib().mgrit_q8_weight_grad_workspace_bytes(rows, _c_int32(out_features), _c_int32(in_features), _DTYPES[dtype]))


def mgrit_q8_weight_grad(dy: torch.Tensor, x: Q8Rows, scale: float = 1.0, dW: Optional[torch.Tensor] = None,
                         db: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None):
    """Returns (dW [out_features, in_features], db [out_features]), fp32, of a linear map whose input rows were kept as x:
    dW = scale * dy^T x, db = scale * the sum of dy's rows.  dy: fp32 or bf16, [..., out_features]."""
    device = _device_of(dy, "dy")
    rows, m, ldy = _check_rows(dy, "dy", device)
    _check_q8(x, "x", device, (*dy.shape[:-1], _is_q8(x, "x").cols))
    handle, other = _on(stream, device)
    if dW is None:
        dW = _new((m, x.cols), torch.float32, dy.device, other)
    else:
        _check_device(dW, "dW", device)
        if dW.dtype != torch.float32 or dW.shape != (m, x.cols) or not dW.is_contiguous():
            raise ValueError(f"dW: expected a contiguous fp32 matrix of shape {(m, x.cols)}, got {dW.dtype} {tuple(dW.shape)}")
    db, db_at = _vector(db, m, "db", device, dy, other)
    L, dtype = lib(), _DTYPES[dy.dtype]
    ws, ws_at, ws_bytes = _workspace(workspace, L.mgrit_q8_weight_grad_workspace_bytes(rows, m, x.cols, dtype), dy.device,
                                     other)
    st = L.mgrit_q8_weight_grad(rows, m, x.cols, dtype, dy.data_ptr(), ldy, x.q.data_ptr(), x.scale.data_ptr(), scale,
                                dW.data_ptr(), db_at, ws_at, ws_bytes, handle)
    if st != MGRIT_OK:
        raise MgritError(st, "mgrit_q8_weight_grad")
    if other is not None:
        _in_use(other, dy, x, dW, db, ws)
    return dW, db
