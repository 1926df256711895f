"""The operators around the layer solves that speed is measured on: the LayerNorm between the last state and the head
of a pre-LayerNorm network, rows kept in 8 bits between the forward and the backward pass, and the gradients that are
taken from such rows.  A case is one call, or one short sequence of calls, of a user's program:

  kind "norm_forward"      y, mean and 1/std of the rows of x
  kind "norm_backward"     dx, dgamma and dbeta from dy, x and the forward pass's statistics
  kind "norm_backward_q8"  the same with x kept as 8-bit rows
  kind "norm_step"         forward with an 8-bit copy of x in the same pass, backward from that copy
  kind "states"            rows to 8 bits and back: what a training step keeps between its two solves
  kind "weight_grad_q8"    dW and db of a linear map whose input was kept as 8-bit rows

8-bit rows: blocks of 32 consecutive elements, the last block of a row filled up with zeros; one power of two 2^e per
block, the smallest with max|x| < 127.5 * 2^e (e >= -126), kept as e + 127; the elements are x * 2^-e rounded to the
nearest integer, ties to even.  A block that holds a NaN, an infinity or the last half percent below it (127.5 * 2^121 and
more) has scale 255 and stands for NaNs.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List, Optional

import torch

own = False                      # True: run() makes the framework's calls, False: the plain form of the same operators
EPS = 1e-5
BLOCK = 32
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def _norm(rows, cols, x, y, pad=0) -> Dict:
    return dict(rows=rows, cols=cols, x=x, y=y, pad=pad)


def listed() -> List[Dict]:
    return [
        # the last LayerNorm for one new token: latency alone
        dict(name="norm_fwd_token", kind="norm_forward", **_norm(1, 768, "fp32", "bf16")),
        # wide rows of a long batch, bf16 throughout
        dict(name="norm_fwd_wide", kind="norm_forward", **_norm(16384, 4096, "bf16", "bf16")),
        # the tiny fp32 encoder (2 x 32 tokens, 64 wide): the smallest backward pass
        dict(name="norm_bwd_tiny", kind="norm_backward", **_norm(64, 64, "fp32", "fp32")),
        # an odd width, rows that are slices of wider ones
        dict(name="norm_bwd_odd", kind="norm_backward", **_norm(5003, 1001, "fp32", "fp32", pad=7)),
        # 64 sequences of 512 tokens at 768 wide, bf16 cotangents from the head, fp32 state
        dict(name="norm_bwd_train", kind="norm_backward", **_norm(32768, 768, "fp32", "bf16")),
        # 64 images of 197 patches at 384 wide, the state kept in 8 bits
        dict(name="norm_bwd_q8_patches", kind="norm_backward_q8", **_norm(12608, 384, "fp32", "bf16")),
        # both passes at the end of a network 2048 wide, 16 sequences of 2048 tokens
        dict(name="norm_step_q8", kind="norm_step", **_norm(32768, 2048, "fp32", "bf16")),
        # the states of the tiny encoder: 17 grid points of 64 tokens
        dict(name="states_tiny", kind="states", **_norm(17 * 64, 64, "fp32", "fp32")),
        # the states of the 128-layer decoder at 768 wide: 129 grid points of 8 x 512 tokens
        dict(name="states_deep", kind="states", **_norm(129 * 4096, 768, "fp32", "fp32")),
        # a feed-forward product of the tiny encoder
        dict(name="weight_grad_tiny", kind="weight_grad_q8", rows=64, out=256, cols=64, y="fp32"),
        # fp32 cotangents (the adjoint states are fp32), ragged tokens and an odd input width
        dict(name="weight_grad_ragged_fp32", kind="weight_grad_q8", rows=12608, out=2048, cols=1000, y="fp32"),
        # a head of 50257 words over 8 x 512 tokens, 768 wide; the largest product
        dict(name="weight_grad_head", kind="weight_grad_q8", rows=4096, out=50257, cols=768, y="bf16"),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random) -> Dict:
    while True:
        kind = rng.choice(["norm_forward", "norm_backward", "norm_backward", "norm_backward_q8", "norm_step", "states",
                           "weight_grad_q8", "weight_grad_q8", "weight_grad_q8"])
        cols = rng.choice([64 * _log_int(rng, 1, 128), 64 * _log_int(rng, 1, 32), _log_int(rng, 8, 6000)])
        rows = _log_int(rng, 1, 65536)
        if rng.random() < 0.3:                       # round lengths are common
            rows = 1 << (rows.bit_length() - 1)
        y = rng.choice(["bf16", "fp32"])
        if kind == "weight_grad_q8":
            out = rng.choice([64 * _log_int(rng, 1, 160), _log_int(rng, 1, 40000)])
            if 2.0 * rows * out * cols * (3 if y == "fp32" else 1) > 3e11 or out * cols > 4e7 or rows * max(out, cols) > 2e8:
                continue
            return dict(kind=kind, rows=rows, out=out, cols=cols, y=y)
        if rows * cols > 6.7e7:
            continue
        x = "fp32" if kind == "norm_step" else rng.choice(["fp32", "fp32", "bf16"])
        pad = rng.choice([0, 0, 0, rng.randint(1, 40)])
        return dict(kind=kind, **_norm(rows, cols, x, x if kind == "states" else y, pad))


# ------------------------------------------------------------------ bytes and flops
def work(case: Dict) -> Dict:
    size = {"fp32": 4.0, "bf16": 2.0}
    n, cols, rows = float(case["rows"]) * case["cols"], case["cols"], case["rows"]
    q8 = rows * 33.0 * ((cols + BLOCK - 1) // BLOCK)
    kind, y = case["kind"], size[case["y"]]
    if kind == "weight_grad_q8":
        out = float(case["out"])
        return {"bytes": rows * out * y + q8 + 4.0 * out * (cols + 1), "flops": 2.0 * rows * out * cols}
    x, vectors, stats = size[case["x"]], 4.0 * cols, 8.0 * rows
    if kind == "norm_forward":
        return {"bytes": n * (x + y) + 2 * vectors + stats, "flops": 8.0 * n}
    if kind == "norm_backward":
        return {"bytes": n * (2 * x + y) + 3 * vectors + stats, "flops": 14.0 * n}
    if kind == "norm_backward_q8":
        return {"bytes": n * (x + y) + q8 + 3 * vectors + stats, "flops": 15.0 * n}
    if kind == "norm_step":                          # the 8-bit copy is written and read
        return {"bytes": n * (2 * x + 2 * y) + 2 * q8 + 5 * vectors + 2 * stats, "flops": 26.0 * n}
    return {"bytes": n * 2 * x + 2 * q8, "flops": 5.0 * n}


# ------------------------------------------------------------------ inputs
def _inputs(case: Dict, seed: int) -> Dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, dtype=torch.float32, device="cuda")

    rows, cols, pad = case["rows"], case["cols"], case.get("pad", 0)
    # every feature has its own spread and offset, a few are far larger than the rest
    x = normal(rows, cols + pad).mul_(torch.exp(0.5 * normal(cols + pad))).add_(0.3 * normal(cols + pad))
    x[:, ::97] *= 20.0
    s = {"x": x.to(TYPES[case.get("x", "fp32")])[:, :cols]}
    if case["kind"] == "weight_grad_q8":
        return dict(s, dy=normal(rows, case["out"]).mul_(0.02).to(TYPES[case["y"]]))
    if case["kind"] == "states":
        return s
    s.update(gamma=1.0 + 0.2 * normal(cols), beta=0.1 * normal(cols))
    if case["kind"] != "norm_forward":
        s.update(dy=normal(rows, cols + pad).mul_(0.02).to(TYPES[case["y"]])[:, :cols])
    return s


def prepare(case: Dict, seed: int) -> Dict:
    s = _inputs(case, seed)
    kind = case["kind"]
    s.update(kind=kind, cols=case["cols"], y_type=TYPES[case["y"]], x_type=s["x"].dtype)
    if kind in ("norm_backward", "norm_backward_q8"):
        s["mean"], s["rstd"] = _statistics(s["x"])
    if kind in ("norm_backward_q8", "weight_grad_q8"):
        s["q"], s["scale"] = _to_q8(s.pop("x"))
    return s


# ------------------------------------------------------------------ the plain forms
def _to_q8(x: torch.Tensor):
    """(q int8 [rows, blocks * 32], scale uint8 [rows, blocks])"""
    rows, cols = x.shape
    blocks = (cols + BLOCK - 1) // BLOCK
    t = torch.zeros((rows, blocks * BLOCK), dtype=torch.float32, device=x.device)
    t[:, :cols] = x
    t = t.view(rows, blocks, BLOCK)
    top = t.abs().view(torch.int32).amax(-1, keepdim=True)         # the bits of a magnitude order like it
    scale = (((top + 0x10000) >> 23) - 6).clamp(min=1)             # one more from 127.5 / 64 on
    q = torch.round(t * ((254 - scale) << 23).view(torch.float32))
    finite = top < 0x7f7f0000                                      # the bits of 127.5 * 2^121
    q = torch.where(finite, q, torch.zeros_like(q)).to(torch.int8)
    scale = torch.where(finite, scale, torch.full_like(scale, 255)).to(torch.uint8)
    return q.view(rows, blocks * BLOCK), scale.view(rows, blocks)


def _from_q8(q: torch.Tensor, scale: torch.Tensor, cols: int) -> torch.Tensor:
    rows, blocks = scale.shape
    step = (scale.to(torch.int32) << 23).view(torch.float32)       # scale 255: infinity, and 0 * infinity = NaN
    return (q.view(rows, blocks, BLOCK).float() * step.view(rows, blocks, 1)).view(rows, blocks * BLOCK)[:, :cols]


def _statistics(x: torch.Tensor):
    x = x.float()
    mean = x.mean(-1, keepdim=True)
    c = x - mean
    return mean[:, 0], torch.rsqrt((c * c).mean(-1) + EPS)


def _norm_forward(x, gamma, beta, y_type):
    mean, rstd = _statistics(x)
    y = (x.float() - mean[:, None]) * rstd[:, None] * gamma + beta
    return y.to(y_type), mean, rstd


def _norm_backward(dy, x, gamma, mean, rstd, x_type):
    dy, xhat = dy.float(), (x.float() - mean[:, None]) * rstd[:, None]
    g, h = dy * gamma, dy * xhat
    dx = rstd[:, None] * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    return dx.to(x_type), h.sum(0), dy.sum(0)


# ------------------------------------------------------------------ one pass
def run(s: Dict) -> Dict:
    kind = s["kind"]
    if own:
        from paper_2601_09026_amd import binding as mb
        if kind == "norm_forward":
            y, mean, rstd = mb.mgrit_layer_norm_forward(s["x"], s["gamma"], s["beta"], eps=EPS, y_dtype=s["y_type"])
            return {"y": y, "mean": mean, "rstd": rstd}
        if kind == "norm_step":
            kept = mb.q8_empty(s["x"].shape, s["x"].device)
            y, mean, rstd = mb.mgrit_layer_norm_forward(s["x"], s["gamma"], s["beta"], eps=EPS, y_dtype=s["y_type"], x_q8=kept)
            dx, dgamma, dbeta = mb.mgrit_layer_norm_backward(s["dy"], kept, s["gamma"], mean, rstd, dx_dtype=s["x_type"])
            return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
        if kind == "states":
            return {"x": mb.mgrit_q8_unpack(mb.mgrit_q8_pack(s["x"]), dtype=s["x_type"])}
        kept = mb.Q8Rows(s["q"], s["scale"], s["cols"]) if "q" in s else s["x"]
        if kind == "weight_grad_q8":
            dW, db = mb.mgrit_q8_weight_grad(s["dy"], kept)
            return {"dW": dW, "db": db}
        dx, dgamma, dbeta = mb.mgrit_layer_norm_backward(s["dy"], kept, s["gamma"], s["mean"], s["rstd"], dx_dtype=s["x_type"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if kind == "norm_forward":
        y, mean, rstd = _norm_forward(s["x"], s["gamma"], s["beta"], s["y_type"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_step":
        q, scale = _to_q8(s["x"])
        y, mean, rstd = _norm_forward(s["x"], s["gamma"], s["beta"], s["y_type"])
        dx, dgamma, dbeta = _norm_backward(s["dy"], _from_q8(q, scale, s["cols"]), s["gamma"], mean, rstd, s["x_type"])
        return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if kind == "states":
        return {"x": _from_q8(*_to_q8(s["x"]), s["cols"]).to(s["x_type"])}
    x = _from_q8(s["q"], s["scale"], s["cols"]) if "q" in s else s["x"]
    if kind == "weight_grad_q8":
        dy = s["dy"].float()
        return {"dW": torch.matmul(dy.t(), x), "db": dy.sum(0)}
    dx, dgamma, dbeta = _norm_backward(s["dy"], x, s["gamma"], s["mean"], s["rstd"], s["x_type"])
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


# ------------------------------------------------------------------ the definition in 64 bits
def _rounded64(x: torch.Tensor) -> torch.Tensor:
    """The values that 8-bit rows of x stand for, from the definition."""
    rows, cols = x.shape
    width = -(-cols // BLOCK) * BLOCK
    t = torch.nn.functional.pad(x.double(), (0, width - cols)).reshape(rows, -1, BLOCK)
    top = t.abs().amax(-1, keepdim=True)
    part, power = torch.frexp(top)                                 # top = part * 2^power, 1/2 <= part < 1
    e = torch.where(part * 128.0 < 127.5, power - 7, power - 6).clamp(min=-126)
    step = ((e.long() + 1023) << 52).view(torch.float64)            # 2^e, exactly
    out = torch.where(top < 127.5 * 2.0 ** 121, torch.round(t / step) * step, torch.full_like(t, math.nan))
    return out.reshape(rows, width)[:, :cols]


def exact(case: Dict, seed: int) -> Optional[Dict]:
    s, kind = _inputs(case, seed), case["kind"]
    x = s["x"].double()
    if kind == "states":
        return {"x": _rounded64(s["x"])}
    if kind == "weight_grad_q8":
        dy = s["dy"].double()
        return {"dW": torch.mm(dy.t().contiguous(), _rounded64(s["x"]).contiguous()), "db": torch.sum(dy, dim=0)}
    gamma = s["gamma"].double()
    var, mean = torch.var_mean(x, dim=1, keepdim=True, correction=0)
    inv = 1.0 / torch.sqrt(var + EPS)
    out = {"y": (x - mean) * inv * gamma + s["beta"].double(), "mean": mean.squeeze(1), "rstd": inv.squeeze(1)}
    if kind == "norm_forward":
        return out
    if kind != "norm_step":
        # the statistics are inputs of the backward pass: as the forward pass left them, in 32 bits
        mean, inv = mean.float().double(), inv.float().double()
    z = ((x if kind == "norm_backward" else _rounded64(s["x"])) - mean) * inv
    dy, n = s["dy"].double(), case["cols"]
    g = dy * gamma
    dx = inv * (g - (g.sum(1, keepdim=True) + z * (g * z).sum(1, keepdim=True)) / n)
    back = {"dx": dx, "dgamma": (dy * z).sum(0), "dbeta": dy.sum(0)}
    return dict(back, y=out["y"]) if kind == "norm_step" else back
