"""The operators between a head's logits and the gradient that enters the network again, that speed is measured on: the log
probabilities of given tokens with entropy and the most likely alternatives, distillation from a teacher's top logits, and
the gradients of both.  A case is one call of a user's program:

  kind "logprobs"           log p of a token per row, the row's entropy and log-sum-exp, its top_k alternatives
  kind "logprobs_backward"  the logits' gradient for given cotangents of the log probabilities and the entropies
  kind "logprobs_step"      both for cotangents that are known beforehand (a mean over tokens): values and gradient
  kind "distill"            sum_j q_j (log q_j - log p_j) per row over a teacher's `kept` top logits
  kind "distill_backward"   its gradient
  kind "distill_step"       both in one call

p = softmax(z / temperature) over a row of `cols` logits z.  q = softmax(y / temperature) over the teacher's kept logits y
whose id is not negative (negative ids fill up shorter lists; a row of such ids has loss and gradient 0).  A token below 0
stands for none: log probability 0 and no gradient through it.  Alternatives are in descending order, ties at the lowest id.
A masked logit is -infinity: its p is 0.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List, Optional

import torch

own = False                      # True: run() makes the framework's calls, False: the plain form of the same operators
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
IDS = {"int64": torch.int64, "int32": torch.int32}


# ------------------------------------------------------------------ the cases
def _rows(rows, cols, dtype, pad=0, temperature=1.0, banned=0.0, masked=0) -> Dict:
    """pad: the rows are slices of wider ones; banned: share of the vocabulary masked at random, row by row; masked: so
    many last columns masked in all rows (a vocabulary filled up to a round width)."""
    return dict(rows=rows, cols=cols, dtype=dtype, pad=pad, temperature=temperature, banned=banned, masked=masked)


def listed() -> List[Dict]:
    return [
        # one new token of a head of 50257 words, with the 20 alternatives that a server reports: latency alone
        dict(name="logprobs_token", kind="logprobs", top_k=20, ids="int64", **_rows(1, 50257, "bf16")),
        # the tokens of 8 prompts of 512, with their 5 best alternatives
        dict(name="logprobs_prompts", kind="logprobs", top_k=5, ids="int64", **_rows(4096, 50257, "bf16")),
        # validation in fp32 over a wide vocabulary, no alternatives
        dict(name="logprobs_wide_fp32", kind="logprobs", top_k=0, ids="int64", **_rows(2048, 131072, "fp32")),
        # an odd vocabulary, slices of wider rows, nine words in ten banned by a grammar, sampled at 0.7
        dict(name="logprobs_banned", kind="logprobs", top_k=20, ids="int32",
             **_rows(777, 32003, "fp32", pad=5, temperature=0.7, banned=0.9)),
        # policy gradients with an entropy bonus: cotangents that depend on the log probabilities
        dict(name="logprobs_bwd_policy", kind="logprobs_backward", entropy=True, ids="int64", **_rows(4096, 50257, "bf16")),
        # 1000 classes of 64 images, fp32: a small backward pass
        dict(name="logprobs_bwd_classes", kind="logprobs_backward", entropy=False, ids="int64", **_rows(64, 1000, "fp32")),
        # cross entropy of a training step, 16 x 512 tokens, the vocabulary filled up to 50304; the largest case
        dict(name="logprobs_step_train", kind="logprobs_step", entropy=False, ids="int64",
             **_rows(8192, 50304, "bf16", masked=47)),
        # masked words of a few sequences
        dict(name="logprobs_step_few", kind="logprobs_step", entropy=False, ids="int64", **_rows(77, 30000, "fp32")),
        # validation against a teacher's 16 best words, ragged lists
        dict(name="distill_ragged", kind="distill", kept=16, ids="int64", values="fp32",
             **_rows(1003, 32003, "fp32", temperature=2.0)),
        # gradient of the same at training size, 64 kept
        dict(name="distill_bwd_train", kind="distill_backward", kept=64, ids="int32", values="bf16",
             **_rows(4096, 50257, "bf16", temperature=2.0)),
        # a tiny classifier's classes: all ten are kept
        dict(name="distill_step_tiny", kind="distill_step", kept=10, ids="int64", values="fp32", **_rows(64, 10, "fp32", temperature=4.0)),
        # a training step against a teacher's 32 best words
        dict(name="distill_step_train", kind="distill_step", kept=32, ids="int64", values="fp32",
             **_rows(4096, 50304, "bf16", temperature=2.0, masked=47)),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random) -> Dict:
    while True:
        kind = rng.choice(["logprobs", "logprobs", "logprobs_backward", "logprobs_step", "distill", "distill_backward", "distill_step"])
        cols = _log_int(rng, 10, 262144)
        if rng.random() < 0.3:                       # round vocabularies are common
            cols = max(64, cols // 64 * 64)
        rows = _log_int(rng, 1, 16384)
        if rng.random() < 0.3:
            rows = 1 << (rows.bit_length() - 1)
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        size = 4 if dtype == "fp32" else 2
        if rows * cols * size > 8.2e8 or rows * cols > 2.7e8:
            continue
        banned = rng.choice([0.0, 0.0, 0.0, 0.5, 0.9]) if cols >= 2000 else 0.0
        masked = rng.randint(1, 63) if cols > 256 and rng.random() < 0.2 else 0
        case = dict(kind=kind, ids=rng.choice(["int64", "int64", "int32"]),
                    **_rows(rows, cols, dtype, rng.choice([0, 0, 0, rng.randint(1, 40)]), rng.choice([1.0, 1.0, 0.7, 2.0]), banned, masked))
        if kind == "logprobs":
            case.update(top_k=rng.choice([k for k in (0, 1, 5, 10, 20, 64) if k <= cols]))
            if case["top_k"] and rows * cols > 2.0e8:
                continue
        elif kind.startswith("logprobs"):
            case.update(entropy=rng.random() < 0.4)
        else:
            case.update(kept=min(cols, rng.choice([1, _log_int(rng, 2, 200), 16, 32, 64])), values=rng.choice(["fp32", "bf16"]))
        return case


# ------------------------------------------------------------------ bytes and flops
def work(case: Dict) -> Dict:
    size = {"fp32": 4.0, "bf16": 2.0, "int64": 8.0, "int32": 4.0}
    rows, n, kind = float(case["rows"]), float(case["rows"]) * case["cols"], case["kind"]
    logits, ids = n * size[case["dtype"]], size[case["ids"]]
    moved = logits if kind in ("logprobs", "distill") else 2.0 * logits
    if kind.startswith("logprobs"):
        row = ids + 12.0 + case.get("top_k", 0) * (ids + 4.0)     # token; three values; alternatives
        row += 0.0 if kind == "logprobs" else 8.0 if case["entropy"] else 4.0
        flops = {"logprobs": 6.0, "logprobs_backward": 6.0, "logprobs_step": 10.0}[kind]
    else:
        row = case["kept"] * (ids + size[case["values"]]) + 8.0
        row += 0.0 if kind == "distill" else 4.0
        flops = {"distill": 4.0, "distill_backward": 4.0, "distill_step": 8.0}[kind]
    return {"bytes": moved + rows * row, "flops": flops * n}


# ------------------------------------------------------------------ inputs
def _statistics(z: torch.Tensor, temperature: float):
    """(log-sum-exp, entropy) of the rows in 64 bits, rounded to 32: what a forward pass hands to the backward pass."""
    lse, entropy = [], []
    for part in z.split(max(1, 2 ** 27 // z.shape[1])):
        y = part.double() / temperature
        top = y.amax(1, keepdim=True)
        e = torch.exp(y - top)
        s = e.sum(1)
        lse.append(top[:, 0] + torch.log(s))
        entropy.append(torch.log(s) - torch.where(e > 0, (y - top) * e, 0.0).sum(1) / s)
    return torch.cat(lse).float(), torch.cat(entropy).float()


def _inputs(case: Dict, seed: int) -> Dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, cols, pad, kind = case["rows"], case["cols"], case["pad"], case["kind"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, dtype=torch.float32, device="cuda")

    # logits of a trained head: frequent and rare words, a few likely ones in each row, the right one often among them
    z = normal(rows, cols + pad).mul_(1.5).add_(1.5 * normal(cols + pad)).sub_(4.0)
    live = cols - case["masked"]
    likely = torch.randint(0, live, (rows, min(8, live)), generator=gen, device="cuda")
    z.scatter_add_(1, likely, 4.0 * normal(*likely.shape).abs_())
    token = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.7, likely[:, 0],
                        torch.randint(0, live, (rows,), generator=gen, device="cuda"))
    if case["banned"]:
        ban = torch.rand(z.shape, generator=gen, device="cuda") < case["banned"]
        ban.scatter_(1, likely, False)
        ban.scatter_(1, token[:, None], False)
        z.masked_fill_(ban, -math.inf)
        del ban
    if case["masked"]:
        z[:, live:cols] = -math.inf
    z = z.to(TYPES[case["dtype"]])[:, :cols]
    s = {"z": z}
    weight = 1.0 / rows * (0.5 + torch.rand(rows, generator=gen, device="cuda"))
    if kind.startswith("logprobs"):
        # one row in twenty is padding
        s["tokens"] = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.05, -100, token).to(IDS[case["ids"]])
        if kind != "logprobs":
            s["g"] = -weight if kind == "logprobs_step" else weight * normal(rows)
            s["h"] = 0.01 * weight if case["entropy"] else None
    else:
        # the teacher sees much the same: its best words, lists of different lengths
        y = z.float() + normal(rows, cols)
        values, ids = torch.topk(y, case["kept"], dim=1)
        del y
        ids = torch.where(torch.isinf(values), -1, ids)
        values = torch.where(torch.isinf(values), 0.0, values)
        length = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.2,
                             torch.randint(0, case["kept"] + 1, (rows,), generator=gen, device="cuda"), case["kept"])
        ids = torch.where(torch.arange(case["kept"], device="cuda") < length[:, None], ids, -1)
        s.update(ids=ids.to(IDS[case["ids"]]), values=values.to(TYPES[case["values"]]), g=weight * case["temperature"] ** 2)
    if kind.endswith("backward"):
        s["lse"], entropy = _statistics(z, case["temperature"])
        if kind.startswith("logprobs"):
            s["entropy"] = entropy if case["entropy"] else None
    return s


def prepare(case: Dict, seed: int) -> Dict:
    return dict(_inputs(case, seed), kind=case["kind"], temperature=case["temperature"], top_k=case.get("top_k", 0))


# ------------------------------------------------------------------ the plain forms
def _softmax(z, temperature):
    """(z / temperature, exp of it less its maximum, the sum of those, log-sum-exp)"""
    y = z.float() / temperature
    top = y.amax(1, keepdim=True)
    e = torch.exp(y - top)
    s = e.sum(1, keepdim=True)
    return y, e, s, top + torch.log(s)


def _alternatives(z, k):
    """Ids of the k largest, ties at the lowest id: unique keys of the value's order and the id's reverse."""
    bits = (z.float() + 0.0).view(torch.int32).long()              # (-0 and 0 are equal)
    order = torch.where(bits < 0, -2 ** 31 - bits, bits)
    key = (order << 32) + torch.arange(z.shape[1] - 1, -1, -1, device=z.device)
    return torch.topk(key, k, dim=1).indices


def _entropy(y, e, s, lse):
    return (lse - torch.where(e > 0, y * e, torch.zeros_like(e)).sum(1, keepdim=True) / s)[:, 0]


def _logprob(y, tokens, lse):
    at = tokens.long().clamp(min=0)[:, None]
    return torch.where(tokens >= 0, (y.gather(1, at) - lse)[:, 0], torch.zeros_like(lse[:, 0]))


def _logprob_gradient(z, temperature, tokens, lse, entropy, g, h):
    lp = z.float() / temperature - lse[:, None]
    p = torch.exp(lp)
    live = tokens >= 0
    g = torch.where(live, g, torch.zeros_like(g))
    d = -g[:, None] * p
    if h is not None:
        d -= h[:, None] * p * (torch.where(p > 0, lp, torch.zeros_like(lp)) + entropy[:, None])
    d.scatter_add_(1, tokens.long().clamp(min=0)[:, None], g[:, None])
    return (d / temperature).to(z.dtype)


def _teacher(ids, values, temperature):
    """(q over the kept, ids with 0 for those left out, 1 for rows with any)"""
    live = ids >= 0
    y = torch.where(live, values.float() / temperature, torch.full(ids.shape, -math.inf, device=ids.device))
    top = y.amax(1, keepdim=True)
    e = torch.exp(y - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(1, keepdim=True)
    some = (total > 0).float()
    return e / torch.where(total > 0, total, torch.ones_like(total)), ids.long().clamp(min=0), some


def _distill_loss(y, lse, q, at):
    terms = q * (torch.log(q) - (y.gather(1, at) - lse))
    return torch.where(q > 0, terms, torch.zeros_like(terms)).sum(1)


def _distill_gradient(z, temperature, lse, q, at, some, g):
    d = torch.exp(z.float() / temperature - lse[:, None]) * some
    d.scatter_add_(1, at, -q)
    return (d * (g[:, None] / temperature)).to(z.dtype)


# ------------------------------------------------------------------ one pass
def run(s: Dict) -> Dict:
    kind, z, temperature = s["kind"], s["z"], s["temperature"]
    if own:
        from paper_2601_09026_amd import binding as mb
        if kind == "logprobs":
            r = mb.mgrit_token_logprobs_forward(z, s["tokens"], top_k=s["top_k"], temperature=temperature)
            out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse}
            return dict(out, top_ids=r.top_ids, top_logprobs=r.top_logprobs) if s["top_k"] else out
        if kind == "logprobs_backward":
            return {"dlogits": mb.mgrit_token_logprobs_backward(z, s["tokens"], s["lse"], s["g"], entropy=s["entropy"], g_entropy=s["h"],
                                                                temperature=temperature)}
        if kind == "logprobs_step":
            r, dlogits = mb.mgrit_token_logprobs_step(z, s["tokens"], s["g"], g_entropy=s["h"], temperature=temperature)
            return {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse, "dlogits": dlogits}
        if kind == "distill":
            loss, lse = mb.mgrit_distill_forward(z, s["ids"], s["values"], temperature=temperature)
            return {"loss": loss, "lse": lse}
        if kind == "distill_backward":
            return {"dlogits": mb.mgrit_distill_backward(z, s["ids"], s["values"], s["lse"], s["g"], temperature=temperature)}
        loss, lse, dlogits = mb.mgrit_distill_step(z, s["ids"], s["values"], s["g"], temperature=temperature)
        return {"loss": loss, "lse": lse, "dlogits": dlogits}
    if kind == "logprobs_backward":
        return {"dlogits": _logprob_gradient(z, temperature, s["tokens"], s["lse"], s["entropy"], s["g"], s["h"])}
    if kind in ("logprobs", "logprobs_step"):
        y, e, total, lse = _softmax(z, temperature)
        entropy = _entropy(y, e, total, lse)
        out = {"logprob": _logprob(y, s["tokens"], lse), "entropy": entropy, "lse": lse[:, 0]}
        if kind == "logprobs_step":
            del e
            out["dlogits"] = _logprob_gradient(z, temperature, s["tokens"], lse[:, 0], entropy, s["g"], s["h"])
        elif s["top_k"]:
            at = _alternatives(z, s["top_k"])
            out.update(top_ids=at.to(s["tokens"].dtype), top_logprobs=y.gather(1, at) - lse)
        return out
    q, at, some = _teacher(s["ids"], s["values"], temperature)
    if kind == "distill_backward":
        return {"dlogits": _distill_gradient(z, temperature, s["lse"], q, at, some, s["g"])}
    y, _, _, lse = _softmax(z, temperature)
    out = {"loss": _distill_loss(y, lse, q, at), "lse": lse[:, 0]}
    if kind == "distill_step":
        out["dlogits"] = _distill_gradient(z, temperature, lse[:, 0], q, at, some, s["g"])
    return out


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_rows(kind: str, s: Dict, tau: float, k: int) -> Dict:
    y = s["z"].double() / tau
    n = torch.arange(y.shape[0], device=y.device)
    out = {}
    if kind.endswith("backward"):
        lse = s["lse"].double()                      # an input, in 32 bits
    else:
        lse = torch.logsumexp(y, dim=1)
        out["lse"] = lse
    lp = y - lse[:, None]
    p = lp.exp()
    if kind.startswith("logprobs"):
        token = s["tokens"].long()
        some = (token >= 0).double()
        token = torch.where(token < 0, torch.zeros_like(token), token)
        if not kind.endswith("backward"):
            entropy = -torch.nan_to_num(p * lp, nan=0.0).sum(1)
            out.update(entropy=entropy, logprob=torch.where(some > 0, lp[n, token], 0.0))
        if kind == "logprobs":
            if k:
                best = torch.sort(s["z"].double(), dim=1, descending=True, stable=True).indices[:, :k]
                out.update(top_ids=best.to(s["tokens"].dtype), top_logprobs=lp.gather(1, best))
            return out
        g = s["g"].double() * some
        d = -g[:, None] * p
        if s["h"] is not None:
            H = s["entropy"].double() if kind.endswith("backward") else entropy
            d -= s["h"].double()[:, None] * torch.nan_to_num(p * (lp + H[:, None]), nan=0.0)
        d[n, token] += g
        return dict(out, dlogits=d / tau)
    ids = s["ids"].long()
    w = torch.where(ids < 0, 0.0, torch.exp(s["values"].double() / tau))
    mass = w.sum(1, keepdim=True)
    q = torch.where(mass > 0, w / mass, 0.0)
    ids = ids.clamp(min=0)
    if kind != "distill_backward":
        out["loss"] = (torch.xlogy(q, q) - torch.where(q > 0, q * lp.gather(1, ids), 0.0)).sum(1)
    if kind != "distill":
        target = torch.zeros_like(p).scatter_add_(1, ids, q)
        out["dlogits"] = (p * (mass > 0) - target) * (s["g"].double() / tau)[:, None]
    return out


def exact(case: Dict, seed: int) -> Optional[Dict]:
    s = _inputs(case, seed)
    step = max(1, 2 ** 26 // case["cols"])           # rows at a time: 64 bits and a sort of them
    parts = [_exact_rows(case["kind"], {k: v if v is None else v[i:i + step] for k, v in s.items()}, case["temperature"],
                         case.get("top_k", 0)) for i in range(0, case["rows"], step)]
    return {name: torch.cat([part[name] for part in parts]) for name in parts[0]}
