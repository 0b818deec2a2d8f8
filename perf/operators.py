"""Operators of the 8-bit forward and of truncated draws, as cases for timing and comparison.

A case is a dict of plain values; `op` names the public entry point:

  add_norm   amd.add_norm_fp8: residual add, RMS norm and gain, e4m3 with a scale per row and block of 128 columns
  quant      amd.quant_fp8: the same rounding of rows that no norm precedes (inputs of the O and down projections)
  gemm       amd.gemm_fp8: product of such rows with e4m3 weights that have a scale per block of 128 x 128; epilogue 0 stores
             (fp32 or bf16), 2 is SiLU * mul of a gate and an up matrix
  sample     amd.sample_rows: temperature, top-k, top-p and min-p, the distribution and a draw by a given uniform

Widths are those of synth.config's pairs.  The plain forms are elementary torch operations; `exact` is the definition in
64 bits, written apart from them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 128                  # columns (and weight rows) that share a scale
E4M3_MAX = 448.0
LEAST = 2.0 ** -100          # a block whose largest magnitude is smaller takes the scale of this one
EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the final norm of a draft step on the 70B shape: one token, all latency
        {"name": "norm_8192_m1", "op": "add_norm", "m": 1, "d": 8192, "h": "fp32", "delta": "fp32"},
        # a 1024-token prompt through the 7B shape (its last token is not part of the prompt pass)
        {"name": "norm_4096_m1023", "op": "add_norm", "m": 1023, "d": 4096, "h": "fp32", "delta": "fp32"},
        # the largest prompt block at the 70B width, residual stream and projection output in bf16
        {"name": "norm_8192_m4096_bf16", "op": "add_norm", "m": 4096, "d": 8192, "h": "bf16", "delta": "bf16"},
        # what the 70B down projection reads in a verify window of 7
        {"name": "quant_28672_m7", "op": "quant", "m": 7, "k": 28672, "x": "bf16"},
        # what the 7B down projection reads in a 2048-token prompt
        {"name": "quant_11008_m2047", "op": "quant", "m": 2047, "k": 11008, "x": "bf16"},
        # the output projection of a 1B-shape draft model: the smallest matrix of a decode step, one token
        {"name": "gemm_2048x2048_m1", "op": "gemm", "m": 1, "n": 2048, "k": 2048, "epilogue": 0, "out": "fp32"},
        # the down projection of the 70B shape over a verify window of 7, for the residual add that follows
        {"name": "gemm_8192x28672_m7", "op": "gemm", "m": 7, "n": 8192, "k": 28672, "epilogue": 0, "out": "bf16"},
        # QKV of the 7B shape for a short prompt or a chunk of one: between the two regimes
        {"name": "gemm_12288x4096_m100", "op": "gemm", "m": 100, "n": 12288, "k": 4096, "epilogue": 0, "out": "bf16"},
        # gate/up of the 70B shape for its 4096-token prompt: the largest single call there is
        {"name": "gemm_57344x8192_m4095", "op": "gemm", "m": 4095, "n": 57344, "k": 8192, "epilogue": 2, "out": "bf16"},
        # a draft step's draw at the pairs' vocabulary with everyday settings
        {"name": "sample_32000_m1", "op": "sample", "rows": 1, "v": 32000, "temperature": 0.75, "top_k": 50, "top_p": 0.9375,
         "min_p": 0.0, "coarse": False},
        # the rows of a verify window of 7 and its bonus row at a large vocabulary: top-p and min-p, no top-k
        {"name": "sample_128256_m8", "op": "sample", "rows": 8, "v": 128256, "temperature": 1.0, "top_k": 0, "top_p": 0.90625,
         "min_p": 0.015625, "coarse": False},
        # many rows whose logits came in bf16, so that equal values meet at every border
        {"name": "sample_128256_m64", "op": "sample", "rows": 64, "v": 128256, "temperature": 1.0, "top_k": 1000,
         "top_p": 0.96875, "min_p": 0.0, "coarse": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _sixteens(rng, lo, hi, step=16):
    return max(step, _log_int(rng, lo, hi) // step * step)


def draw(rng):
    op = rng.choice(["add_norm", "quant", "gemm", "gemm", "sample", "sample"])
    if op == "add_norm":
        h, delta = rng.choice([("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "none"), ("bf16", "fp32")])
        return {"op": op, "m": _log_int(rng, 1, 4096), "d": _sixteens(rng, 256, 16384), "h": h, "delta": delta}
    if op == "quant":
        return {"op": op, "m": _log_int(rng, 1, 4096), "k": _sixteens(rng, 256, 28672), "x": rng.choice(["bf16", "bf16", "fp32"])}
    if op == "gemm":
        epilogue, out = rng.choice([(0, "fp32"), (0, "bf16"), (0, "bf16"), (2, "bf16")])
        m = rng.choice([_log_int(rng, 1, 32), _log_int(rng, 1, 4096)])
        n = _sixteens(rng, 256, 57344, 32 if epilogue == 2 else 16)
        return {"op": op, "m": m, "n": n, "k": _sixteens(rng, 256, 8192 if n > 16384 else 28672), "epilogue": epilogue, "out": out}
    return {"op": op, "rows": _log_int(rng, 1, 48), "v": _log_int(rng, 1000, 160000), "temperature": rng.choice([0.5, 0.75, 1.0, 1.5]),
            "top_k": rng.choice([0, 0, _log_int(rng, 1, 2000)]), "top_p": rng.choice([1.0, rng.randint(16, 63) / 64]),
            "min_p": rng.choice([0.0, 0.0, rng.randint(1, 16) / 128]), "coarse": rng.choice([False, True])}


# ---- inputs ----------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, m, k):
    """Rows as a forward has them: a few columns are an order of magnitude above the rest."""
    x = _normal(g, m, k)
    return x * torch.where(torch.rand(k, generator=g, device="cuda") < 0.01, 12.0, 1.0)


def _weight(g, n, k):
    """e4m3 [n][k] and the scales [ceil(n / 128)][ceil(k / 128)] of N(0, 0.02^2)."""
    q = torch.empty(n, k, dtype=torch.float8_e4m3fn, device="cuda")
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    scale = torch.empty(nb, kb, dtype=torch.float32, device="cuda")
    rows = max(BLOCK, (1 << 26) // k // BLOCK * BLOCK)
    for i in range(0, n, rows):
        w = _normal(g, min(rows, n - i), k) * 0.02
        blocks = torch.zeros(-(-w.shape[0] // BLOCK) * BLOCK, kb * BLOCK, device="cuda")
        blocks[: w.shape[0], :k] = w
        blocks = blocks.view(-1, BLOCK, kb, BLOCK)
        s = blocks.abs().amax(dim=(1, 3)).clamp_min(LEAST) / E4M3_MAX
        scale[i // BLOCK : i // BLOCK + s.shape[0]] = s
        q[i : i + w.shape[0]] = (blocks / s[:, None, :, None]).reshape(-1, kb * BLOCK)[: w.shape[0], :k].to(torch.float8_e4m3fn)
    return q, scale


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    if op == "add_norm":
        m, d = case["m"], case["d"]
        s = {"h": _activations(g, m, d).to(TYPES[case["h"]]), "gain": (1 + 0.3 * _normal(g, d)).to(torch.bfloat16)}
        s["delta"] = None if case["delta"] == "none" else (0.3 * _normal(g, m, d)).to(TYPES[case["delta"]])
    elif op == "quant":
        s = {"x": _activations(g, case["m"], case["k"]).to(TYPES[case["x"]])}
    elif op == "gemm":
        m, n, k, epilogue = case["m"], case["n"], case["k"], case["epilogue"]
        q, scale = _quantize(_activations(g, m, k))
        s = {"x": q, "x_scale": scale}
        s["weights"] = [_weight(g, n // 2, k), _weight(g, n // 2, k)] if epilogue == 2 else [_weight(g, n, k)]
    else:
        rows, v = case["rows"], case["v"]
        logits = 2.5 * _normal(g, rows, v)                  # a tail of small ids, and a few that stand out
        top = (torch.randint(v, (rows, 1), generator=g, device="cuda") + torch.arange(24, device="cuda") * (v // 24)) % v
        logits.scatter_(1, top, 6 + 3 * _normal(g, rows, 24))
        s = {"logits": logits.to(torch.bfloat16).float() if case["coarse"] else logits,
             "u": torch.rand(rows, generator=g, device="cuda")}
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2408_11850_amd as amd

        s["amd"] = amd
        amd.load_library()
        if case["op"] == "gemm":                            # weights are laid out once, when a model is loaded
            s["packed"] = amd.pack_weights_fp8(s.pop("weights"), interleave=case["epilogue"] == 2)
    return s


# ---- one pass --------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        amd = state["amd"]
        if op == "add_norm":
            q, scale = amd.add_norm_fp8(state["h"], state["delta"], state["gain"], EPS)
            return {"h": state["h"], "q": q, "scale": scale}
        if op == "quant":
            q, scale = amd.quant_fp8(state["x"])
            return {"q": q, "scale": scale}
        if op == "gemm":
            return amd.gemm_fp8(state["x"], state["x_scale"], state["packed"], case["epilogue"], TYPES[case["out"]])
        tokens, q = amd.sample_rows(state["logits"], state["u"], case["temperature"], 1.0, case["top_k"], case["top_p"],
                                    case["min_p"])
        return {"tokens": tokens, "q": q}
    if op == "add_norm":
        return _plain_add_norm(state)
    if op == "quant":
        q, scale = _quantize(state["x"].float())
        return {"q": q, "scale": scale}
    if op == "gemm":
        return _plain_gemm(state, case["epilogue"], TYPES[case["out"]])
    return _plain_sample(state, case)


def _quantize(y):
    """e4m3 [m][k] and scales [ceil(k / 128)][m] of fp32 rows."""
    m, k = y.shape
    blocks = torch.nn.functional.pad(y, (0, -k % BLOCK)).view(m, -1, BLOCK)
    scale = blocks.abs().amax(dim=2).clamp_min(LEAST) / E4M3_MAX
    q = (blocks / scale[:, :, None]).view(m, -1)[:, :k].to(torch.float8_e4m3fn)
    return q.contiguous(), scale.t().contiguous()


def _plain_add_norm(s):
    h = s["h"]
    if s["delta"] is not None:
        h.copy_(h.float() + s["delta"].float())             # in place; the norm is that of what is stored
    x = h.float()
    y = x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + EPS) * s["gain"].float()
    q, scale = _quantize(y)
    return {"h": h, "q": q, "scale": scale}


def _spread(scale, n, k):
    """A scale per block of 128 x 128, one per element."""
    return scale.repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]


def _plain_gemm(s, epilogue, out):
    m, k = s["x"].shape
    x = s["x"].float() * s["x_scale"].t().repeat_interleave(BLOCK, 1)[:, :k]
    y = [x @ (q.float() * _spread(scale, q.shape[0], k)).t() for q, scale in s["weights"]]
    if epilogue == 2:
        return (y[0] / (1 + torch.exp(-y[0])) * y[1]).to(out)
    return y[0].to(out)


def _plain_sample(s, case):
    """In 64 bits: which id is the last to be kept, and which one a uniform meets, is decided next to borders."""
    z = s["logits"].double() / case["temperature"]
    v = z.shape[1]
    w = torch.exp(z - z.amax(dim=1, keepdim=True))
    sorted_w, ids = torch.sort(z, dim=1, descending=True, stable=True)       # equal values: the lowest id first
    sorted_w = w.gather(1, ids)
    if 0 < case["top_k"] < v:
        sorted_w[:, case["top_k"] :] = 0
    if case["top_p"] < 1:
        before = sorted_w.cumsum(1) - sorted_w
        sorted_w = torch.where(before < case["top_p"] * sorted_w.sum(1, keepdim=True), sorted_w, 0.0)
    sorted_w = torch.where(sorted_w >= case["min_p"], sorted_w, 0.0)
    w = torch.zeros_like(w).scatter_(1, ids, sorted_w)
    cdf = w.cumsum(1)
    total = cdf[:, -1:]
    tokens = (cdf <= s["u"].double()[:, None] * total).sum(1).clamp_max(v - 1).to(torch.int32)
    return {"tokens": tokens, "q": (w / total).float()}


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    op = case["op"]
    size = {"fp32": 4, "bf16": 2, "none": 0}
    if op == "add_norm":
        m, d = case["m"], case["d"]
        h = size[case["h"]] * (1 if case["delta"] == "none" else 2)
        return {"bytes": m * d * (h + size[case["delta"]] + 1) + 4 * m * -(-d // BLOCK) + 2 * d, "flops": 8 * m * d}
    if op == "quant":
        m, k = case["m"], case["k"]
        return {"bytes": m * k * (size[case["x"]] + 1) + 4 * m * -(-k // BLOCK), "flops": 3 * m * k}
    if op == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // BLOCK)
        out = m * n * size[case["out"]] // (2 if case["epilogue"] == 2 else 1)
        return {"bytes": n * k + 4 * -(-n // BLOCK) * kb + m * k + 4 * m * kb + out, "flops": 2 * m * n * k}
    return {"bytes": case["rows"] * (8 * case["v"] + 8), "flops": 20 * case["rows"] * case["v"]}


# ---- the definitions in 64 bits --------------------------------------------------------------
def _e4m3(v):
    """Nearest value with 4 significant bits (3 below 2^-6), ties to the even one, at most 448."""
    exponent = torch.frexp(v)[1].to(torch.float64) - 1
    step = torch.exp2(exponent.clamp_min(-6.0) - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_blocks(y):
    q, scale = torch.empty_like(y), []
    for b in range(0, y.shape[1], BLOCK):
        part = y[:, b : b + BLOCK]
        s = torch.maximum(part.abs().max(dim=1).values, torch.tensor(LEAST, dtype=torch.float64, device=y.device)) / E4M3_MAX
        q[:, b : b + BLOCK] = _e4m3(part / s[:, None])
        scale.append(s)
    return {"q": q, "scale": torch.stack(scale)}


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "quant":
        return _exact_blocks(s["x"].double())
    if op == "add_norm":
        h = s["h"].double()
        if s["delta"] is not None:
            h = (h + s["delta"].double()).to(s["h"].dtype).double()
        y = h / torch.sqrt((h * h).sum(dim=1, keepdim=True) / h.shape[1] + EPS) * s["gain"].double()
        return {"h": h, **_exact_blocks(y)}
    if op == "gemm":
        m, k = s["x"].shape
        y = []
        for q, scale in s["weights"]:
            out = torch.empty(m, q.shape[0], dtype=torch.float64, device="cuda")
            for i in range(0, q.shape[0], 64 * BLOCK):      # so many weight rows at a time in 64 bits
                w = q[i : i + 64 * BLOCK].double()
                for b in range(0, k, BLOCK):
                    rows = torch.arange(i, i + w.shape[0], device="cuda") // BLOCK
                    w[:, b : b + BLOCK] *= scale[rows, b // BLOCK].double()[:, None]
                x = s["x"].double()
                for b in range(0, k, BLOCK):
                    x[:, b : b + BLOCK] *= s["x_scale"][b // BLOCK].double()[:, None]
                out[:, i : i + w.shape[0]] = torch.mm(x, w.t().contiguous())
            y.append(out)
        if case["epilogue"] == 2:
            return y[0] * torch.sigmoid(y[0]) * y[1]
        return y[0]
    tokens, q = [], []
    for row, u in zip(s["logits"].cpu().numpy().astype(np.float64), s["u"].cpu().numpy().astype(np.float64)):
        w = np.exp((row - row.max()) / case["temperature"])
        order = np.lexsort((np.arange(row.size), -row))
        if 0 < case["top_k"] < row.size:
            order = order[: case["top_k"]]
        if case["top_p"] < 1:
            reached = np.cumsum(w[order])
            order = order[: int(np.searchsorted(reached, case["top_p"] * w[order].sum())) + 1]
        kept = np.zeros_like(w)
        kept[order] = w[order]
        kept[kept < case["min_p"]] = 0
        cdf = np.cumsum(kept)
        tokens.append(min(int(np.searchsorted(cdf, u * cdf[-1], side="right")), int(np.flatnonzero(kept)[-1])))
        q.append(kept / cdf[-1])
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "q": torch.from_numpy(np.stack(q))}
