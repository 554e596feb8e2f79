"""Operators that work on whole sets of rows around the SGD chains, each in its plain form and through the library's entry points:

  quantize   rows -> 8-bit rows (e4m3) with a scale for each block of 128 columns
  margins    Z = X W^T: the margins of many models on many rows, both held in 8 bits with block scales
  gradient   objective, 0/1 error and gradient of the objective over all rows, of fp32, bf16 or 8-bit rows
  clip       global norm of a list of gradients, and the gradients scaled down to a given norm

A case names sizes, types and hyper-parameters. `prepare` makes the inputs on the GPU from a seed, `run` is one pass.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128          # columns that share a scale
E4M3_MAX = 448.0     # largest finite value of e4m3
AMAX_MIN = 2.0 ** -100  # blocks whose largest magnitude is below this are scaled as if it were this
LOSSES = {"hinge": 0, "logistic": 1, "squared": 2}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # a test set as it comes from a file, with an odd number of columns: the last block is short and no row but the first aligned
        {"name": "quantize_odd_f32", "op": "quantize", "rows": 4096, "d": 999, "dtype": "f32"},
        # the rows of some nodes of the headline configuration, packed once for all later passes
        {"name": "quantize_wide_bf16", "op": "quantize", "rows": 131072, "d": 4096, "dtype": "bf16"},
        # one new row answered by a thousand models: latency counts
        {"name": "margins_one_row", "op": "margins", "rows": 1, "d": 256, "models": 1024, "out": "f32"},
        # a small ragged batch on an odd number of models
        {"name": "margins_odd_bf16", "op": "margins", "rows": 2047, "d": 999, "models": 37, "out": "bf16"},
        # a large test set on the models of a few nodes: bound by the rows
        {"name": "margins_few_models", "op": "margins", "rows": 262144, "d": 4096, "models": 16, "out": "f32"},
        # a test set on every model of a cluster of a thousand nodes with wide rows: bound by the products
        {"name": "margins_many_models", "op": "margins", "rows": 65536, "d": 4096, "models": 1024, "out": "f32"},
        # the smallest full gradient: one shard of narrow rows, latency counts
        {"name": "gradient_tiny_f32", "op": "gradient", "rows": 4096, "d": 64, "dtype": "f32", "loss": "hinge"},
        # all rows of a few nodes of the headline configuration
        {"name": "gradient_wide_bf16", "op": "gradient", "rows": 262144, "d": 4096, "dtype": "bf16", "loss": "logistic"},
        # 8-bit rows with an odd number of columns
        {"name": "gradient_odd_e4m3", "op": "gradient", "rows": 131072, "d": 999, "dtype": "e4m3", "loss": "squared"},
        # gradients of a few nodes: latency counts
        {"name": "clip_few_f32", "op": "clip", "tensors": 16, "size": 1024, "ragged": False, "dtype": "f32", "clips": True},
        # many small half-precision gradients of unequal sizes, packed one behind the other
        {"name": "clip_many_bf16", "op": "clip", "tensors": 1024, "size": 4096, "ragged": True, "dtype": "bf16", "clips": True},
        # gradients of nodes with a million columns
        {"name": "clip_large_f32", "op": "clip", "tensors": 64, "size": 1 << 20, "ragged": False, "dtype": "f32", "clips": True},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm; odd ones as often as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "margins", "margins", "gradient", "gradient", "clip"])
    if op == "quantize":
        d = _spread(rng, 16, 8192)
        return {"op": op, "rows": _spread(rng, 1, max(1, min(262144, (1 << 29) // d))), "d": d, "dtype": rng.choice(["f32", "bf16"])}
    if op == "margins":
        d, models = _spread(rng, 16, 8192), _spread(rng, 1, 1024)
        rows = _spread(rng, 1, max(1, min(262144, (1 << 30) // d, (1 << 38) // (d * models))))
        return {"op": op, "rows": rows, "d": d, "models": models, "out": rng.choice(["f32", "bf16"])}
    if op == "gradient":
        d = _spread(rng, 8, 8192)
        return {"op": op, "rows": _spread(rng, 1, max(1, min(1 << 20, (1 << 29) // d))), "d": d, "dtype": rng.choice(["f32", "bf16", "e4m3"]),
                "loss": rng.choice(["hinge", "logistic", "squared"])}
    tensors = _spread(rng, 1, 2048)
    return {"op": op, "tensors": tensors, "size": _spread(rng, 16, max(16, (1 << 26) // tensors)), "ragged": rng.random() < 0.5,
            "dtype": rng.choice(["f32", "bf16"]), "clips": rng.random() < 0.8}


# ---- inputs --------------------------------------------------------------------------------------------------------------
def _blocks(d):
    return -(-d // BLOCK)


def _sizes(case):
    n, size = case["tensors"], case["size"]
    return [size - (i * 37) % (size // 2 + 1) if case["ragged"] else size for i in range(n)]


def _packed(rows, d):
    """Storage of 8-bit rows as the library takes them: rows start on 16 bytes."""
    return torch.zeros(rows, (d + 15) // 16 * 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :d]


def _pack(x):
    """8-bit rows and scales of fp32 rows, made here so that they do not depend on any code under measurement."""
    rows, d = x.shape
    a = torch.nn.functional.pad(x, (0, _blocks(d) * BLOCK - d)).view(rows, -1, BLOCK).abs().amax(2).clamp_min(AMAX_MIN)
    q = _packed(rows, d)
    q.copy_((x * (E4M3_MAX / a).repeat_interleave(BLOCK, 1)[:, :d]).to(torch.float8_e4m3fn))
    return q, a / E4M3_MAX


def _normal(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _rows(rows, d, gen):
    """Rows of about unit length whose columns differ in size, as features do: row by row some are several times the usual length."""
    x = _normal((rows, d), gen, torch.float32)
    x *= torch.exp(0.5 * _normal((1, d), gen)) / math.sqrt(d)
    x *= torch.exp(0.3 * _normal((rows, 1), gen))
    return x


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 17)
    op = case["op"]
    s = {"case": case, "op": op, "ctx": None}
    if op == "quantize":
        s["x"] = _rows(case["rows"], case["d"], gen).to(DTYPES[case["dtype"]])
    elif op == "margins":
        s["q"], s["q_scales"] = _pack(_rows(case["rows"], case["d"], gen))
        s["m"], s["m_scales"] = _pack(_normal((case["models"], case["d"]), gen) * torch.exp(0.5 * _normal((case["models"], 1), gen)))
    elif op == "gradient":
        rows, d = case["rows"], case["d"]
        x = _rows(rows, d, gen)
        truth = _normal((d,), gen)
        score = x @ truth + 0.3 * _normal((rows,), gen)
        s["y"] = score if case["loss"] == "squared" else torch.where(score >= 0, 1.0, -1.0)
        s["w"] = 0.7 * truth + 0.3 * _normal((d,), gen)  # on the way to the optimum, not there
        s["lam"] = 1e-4
        if case["dtype"] == "e4m3":
            s["x"], s["scales"] = _pack(x)
        else:
            s["x"], s["scales"] = x.to(DTYPES[case["dtype"]]), None
    else:
        sizes = _sizes(case)
        size_of = torch.tensor(sizes, device="cuda")
        levels = torch.exp(1.5 * _normal((len(sizes),), gen) - 4.0)
        g = _normal((sum(sizes),), gen) * torch.repeat_interleave(levels, size_of)
        s["flat"] = g.to(DTYPES[case["dtype"]])
        s["flat_out"] = torch.zeros_like(s["flat"])
        s["grads"], s["outs"] = list(s["flat"].split(sizes)), list(s["flat_out"].split(sizes))
        expected = math.sqrt(float((levels.double().square() * size_of).sum()))
        s["max_norm"] = 0.25 * expected if case["clips"] else 4.0 * expected
    if own:
        import paper_1708_04801_b200 as P

        s["ctx"] = P.Context(case.get("models", 1), case.get("d", 1))
        if op == "clip":
            s["list"] = P.GradList(s["grads"], s["outs"])
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------
def _widen(q, scales):
    """fp32 values of 8-bit rows."""
    return q.float() * scales.repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _quantize(s):
    if own:
        q, scales = s["ctx"].quantize_rows(s["x"])
        return {"q": q, "scales": scales}
    x = s["x"].float()
    d = x.shape[1]
    a = torch.nn.functional.pad(x, (0, _blocks(d) * BLOCK - d)).view(x.shape[0], -1, BLOCK).abs().amax(2).clamp_min(AMAX_MIN)
    q = x * (E4M3_MAX / a).repeat_interleave(BLOCK, 1)[:, :d]
    return {"q": q.to(torch.float8_e4m3fn), "scales": a / E4M3_MAX}


def _margins(s):
    dtype = DTYPES[s["case"]["out"]]
    if own:
        return s["ctx"].margins_fp8(s["q"], s["q_scales"], s["m"], s["m_scales"], dtype=dtype)
    return torch.matmul(_widen(s["q"], s["q_scales"]), _widen(s["m"], s["m_scales"]).t()).to(dtype)


def _gradient(s):
    loss = s["case"]["loss"]
    if own:
        if s["scales"] is not None:
            out, grad = s["ctx"].objective_grad_fp8(s["x"], s["scales"], s["y"], s["w"], s["lam"], LOSSES[loss])
        else:
            out, grad = s["ctx"].objective_grad(s["x"], s["y"], s["w"], s["lam"], LOSSES[loss])
        return {"measures": out, "grad": grad}
    x = s["x"].float() if s["scales"] is None else _widen(s["x"], s["scales"])
    y, w, lam, n = s["y"].double(), s["w"].double(), s["lam"], s["x"].shape[0]
    z = torch.mv(x.double(), w)  # in 64 bits: hinge losses and signs of margins next to the border
    if loss == "hinge":
        value, g = (1.0 - y * z).clamp_min(0.0), torch.where(y * z < 1.0, -y, torch.zeros_like(y))
    elif loss == "logistic":
        value, g = torch.logaddexp(torch.zeros_like(z), -y * z), -y / (1.0 + torch.exp(y * z))
    else:
        value, g = 0.5 * (z - y).square(), z - y
    wrong = ((z >= 0) != (y >= 0)).double()
    measures = torch.stack([0.5 * lam * w.square().sum() + value.mean(), wrong.mean()]).float()
    grad = torch.mv(x.t(), g.float()) / n + lam * s["w"]
    return {"measures": measures, "grad": grad}


def _clip(s):
    if own:
        norm = s["ctx"].clip_grad_norm(s["list"], s["max_norm"])
        return {"norm": norm, "grads": s["flat_out"]}
    norm = s["flat"].float().square().sum(dtype=torch.float64).sqrt()  # in 64 bits: a long sum
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    return {"norm": norm.float().reshape(1), "grads": (s["flat"].float() * factor).to(s["flat"].dtype)}


def run(state):
    return {"quantize": _quantize, "margins": _margins, "gradient": _gradient, "clip": _clip}[state["op"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "clip":
        n, es = sum(_sizes(case)), 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * n * es + 4, "flops": 3 * n}
    rows, d = case["rows"], case["d"]
    nb = _blocks(d)
    if op == "quantize":
        return {"bytes": rows * (d * (4 if case["dtype"] == "f32" else 2) + d + 4 * nb), "flops": 3 * rows * d}
    if op == "margins":
        m = case["models"]
        return {"bytes": (rows + m) * (d + 4 * nb) + rows * m * (4 if case["out"] == "f32" else 2), "flops": 2 * rows * m * d}
    row = {"f32": 4 * d, "bf16": 2 * d, "e4m3": d + 4 * nb}[case["dtype"]]
    return {"bytes": rows * (row + 4) + 8 * d + 8, "flops": 4 * rows * d}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------
def _scale_of_columns(scales, d):
    column = torch.arange(d, device=scales.device)
    return scales.double()[:, torch.div(column, BLOCK, rounding_mode="floor")]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x = s["x"]
        rows, d = x.shape
        scales = torch.empty(rows, _blocks(d), dtype=torch.float64, device=x.device)
        for b in range(_blocks(d)):
            scales[:, b] = x[:, b * BLOCK:(b + 1) * BLOCK].double().abs().max(dim=1).values.clamp(min=AMAX_MIN) / E4M3_MAX
        return {"q": None, "scales": scales}  # a rounding to 8 bits has no value in 64
    if op == "margins":
        rows, m, d = case["rows"], case["models"], case["d"]
        w = s["m"].double() * _scale_of_columns(s["m_scales"], d)
        z = torch.empty(rows, m, dtype=torch.float64, device=w.device)
        for at in range(0, rows, 16384):
            part = slice(at, min(rows, at + 16384))
            z[part] = (s["q"][part].double() * _scale_of_columns(s["q_scales"][part], d)) @ w.t()
        return z
    if op == "gradient":
        rows, d, loss = case["rows"], case["d"], case["loss"]
        w = s["w"].double()
        total, wrong, grad = 0.0, 0, torch.zeros(d, dtype=torch.float64, device=w.device)
        for at in range(0, rows, 32768):
            part = slice(at, min(rows, at + 32768))
            x, y = s["x"][part].double(), s["y"][part].double()
            if s["scales"] is not None:
                x = x * _scale_of_columns(s["scales"][part], d)
            z = x @ w
            if loss == "squared":
                total += float(((z - y) ** 2).sum()) / 2
                g = z - y
            elif loss == "logistic":
                total += float(torch.nn.functional.softplus(-y * z, threshold=1e9).sum())
                g = -y * torch.sigmoid(-y * z)
            else:
                total += float(torch.relu(1 - y * z).sum())
                g = -y * (1 - y * z > 0).double()
            wrong += int(((z < 0) != (y < 0)).sum())
            grad += x.t() @ g
        measures = torch.tensor([s["lam"] / 2 * float(w @ w) + total / rows, wrong / rows], dtype=torch.float64)
        return {"measures": measures, "grad": grad / rows + s["lam"] * w}
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / norm)
    return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": s["flat"].double() * factor}
