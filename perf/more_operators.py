"""Operators for rows that go to several nodes and for chains whose labels are vectors, each in its plain form and through the library's entry points:

  dispatch   rows sorted by the nodes they are assigned to: shard offsets, positions, and the rows themselves in that order
  combine    what the nodes give for their rows, brought back to the rows' order and added up with a weight for each node
  regrad     the gradients of combine: of the nodes' rows and of the weights
  chain      gated delta rule: each head of a chain keeps dv linear models on dk features, and every row decays them, takes one
             squared-loss step towards its value, and is answered by them
  chaingrad  the same for training: the answers, and the gradients of everything that went in
  step       one row for each of many chains, on models that stay where they are: the form that serves

A case names sizes and types. `prepare` makes the inputs on the GPU from a seed, `run` is one pass.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64                      # rows that the plain form of a chain takes at once
SPEEDS = (1.0, 0.7, 0.4, 0.1)   # relative lengths of the chains: nodes of four speeds in turn


def listed():
    return [
        # a small batch of rows on a few nodes, two nodes a row: latency counts
        {"name": "dispatch_few_f32", "op": "dispatch", "rows": 64, "d": 1024, "nodes": 16, "top": 2, "dtype": "f32", "dropped": False},
        # the rows of a cluster of the headline configuration laid out by node, each on two of 128 nodes
        {"name": "dispatch_wide_bf16", "op": "dispatch", "rows": 65536, "d": 4096, "nodes": 128, "top": 2, "dtype": "bf16", "dropped": False},
        # a ragged batch with an odd number of columns, some of whose places are padding
        {"name": "combine_odd_bf16", "op": "combine", "rows": 2047, "d": 999, "nodes": 37, "top": 3, "dtype": "bf16", "dropped": True},
        # a large batch of fp32 rows back from a thousand nodes
        {"name": "combine_wide_f32", "op": "combine", "rows": 131072, "d": 1024, "nodes": 1024, "top": 4, "dtype": "f32", "dropped": False},
        # a small step of training: latency counts
        {"name": "regrad_few_f32", "op": "regrad", "rows": 333, "d": 1000, "nodes": 16, "top": 2, "dtype": "f32", "dropped": True},
        # a large step of training on wide half-precision rows
        {"name": "regrad_wide_bf16", "op": "regrad", "rows": 65536, "d": 4096, "nodes": 128, "top": 2, "dtype": "bf16", "dropped": False},
        # short fp32 chains that go on from models they have
        {"name": "chain_short_f32", "op": "chain", "rows": 333, "chains": 8, "hk": 4, "hv": 4, "dk": 64, "dv": 48, "dtype": "f32", "start": True},
        # long chains of four speeds, two heads of values to each head of features
        {"name": "chain_long_bf16", "op": "chain", "rows": 65536, "chains": 16, "hk": 8, "hv": 16, "dk": 128, "dv": 128, "dtype": "bf16", "start": False},
        # a small step of training with sizes that fit no tile
        {"name": "chaingrad_odd_bf16", "op": "chaingrad", "rows": 1021, "chains": 5, "hk": 3, "hv": 3, "dk": 60, "dv": 33, "dtype": "bf16"},
        # a large step of training
        {"name": "chaingrad_long_bf16", "op": "chaingrad", "rows": 32768, "chains": 16, "hk": 8, "hv": 16, "dk": 128, "dv": 128, "dtype": "bf16"},
        # one new row for each of four chains: latency counts
        {"name": "step_few_f32", "op": "step", "chains": 4, "pool": 6, "hk": 4, "hv": 4, "dk": 64, "dv": 64, "dtype": "f32"},
        # one new row for each of many chains: bound by the models
        {"name": "step_many_bf16", "op": "step", "chains": 256, "pool": 300, "hk": 16, "hv": 32, "dk": 128, "dv": 128, "dtype": "bf16"},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm; odd ones as often as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    op = rng.choice(["dispatch", "combine", "regrad", "chain", "chain", "chaingrad", "chaingrad", "step"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("dispatch", "combine", "regrad"):
        nodes = _spread(rng, 1, 2048)
        top = min(nodes, _spread(rng, 1, 8))
        d = _spread(rng, 8, 8192)
        rows = _spread(rng, 1, max(1, min(1 << 18, (1 << 27) // (d * top))))
        return {"op": op, "rows": rows, "d": d, "nodes": nodes, "top": top, "dtype": dtype, "dropped": rng.random() < 0.4}
    hk = _spread(rng, 1, 8)
    hv = hk * rng.choice([1, 1, 2, 3])
    dk, dv = _spread(rng, 16, 128), _spread(rng, 16, 128)
    if rng.random() < 0.5:
        dk, dv = rng.choice([32, 64, 128]), rng.choice([32, 64, 128])
    if op == "step":
        chains = _spread(rng, 1, max(1, (1 << 26) // (hv * dk * dv)))
        return {"op": op, "chains": chains, "pool": chains + rng.randrange(0, 1 + chains // 4), "hk": hk, "hv": hv, "dk": dk, "dv": dv, "dtype": dtype}
    chains = _spread(rng, 1, 64)
    if op == "chaingrad":
        rows = _spread(rng, chains, max(chains, min(16384, 2 * chains * 1024, (1 << 25) // (hv * max(dk, dv)))))
        return {"op": op, "rows": rows, "chains": chains, "hk": hk, "hv": hv, "dk": dk, "dv": dv, "dtype": "bf16"}
    most = 65536 if dtype == "bf16" else 4096
    rows = _spread(rng, chains, max(chains, min(most, 2 * chains * 1024, (1 << 26) // (hv * max(dk, dv)))))
    return {"op": op, "rows": rows, "chains": chains, "hk": hk, "hv": hv, "dk": dk, "dv": dv, "dtype": dtype, "start": rng.random() < 0.5}


# ---- inputs --------------------------------------------------------------------------------------------------------------
def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _assign(case, gen):
    """Distinct nodes for each row, some nodes liked far more than others; -1 where a place is padding."""
    liked = 1.5 * _normal((1, case["nodes"]), gen)
    noise = torch.rand((case["rows"], case["nodes"]), generator=gen, device="cuda").clamp_(1e-7, 1 - 1e-7)
    node = (liked - torch.log(-torch.log(noise))).topk(case["top"], dim=1).indices.to(torch.int32)
    if case["dropped"]:
        padding = torch.rand((case["rows"], 1), generator=gen, device="cuda") < 0.1                  # whole rows of padding
        full = torch.rand((case["rows"], case["top"]), generator=gen, device="cuda") < 0.05        # nodes that take no more
        node[padding | full] = -1
    return node.contiguous()


def _positions(node):
    """Where each place's row stands among the rows sorted by node (-1: nowhere), in the order of the rows within a node."""
    flat = node.reshape(-1).long()
    order = torch.argsort(torch.where(flat < 0, torch.full_like(flat, 1 << 40), flat), stable=True)
    where = torch.empty_like(order)
    where[order] = torch.arange(order.numel(), device=order.device)
    return torch.where(flat < 0, torch.full_like(where, -1), where).to(torch.int32).view(node.shape), order


def _lengths(case):
    """Rows of each chain: as its speed among all, the remainder to the first ones."""
    n, speeds = case["rows"], [SPEEDS[c % 4] for c in range(case["chains"])]
    got = [int(n * s / sum(speeds)) for s in speeds]
    left = n - sum(got)
    return [x + left // len(got) + (1 if c < left % len(got) else 0) for c, x in enumerate(got)]


def _rows_of_chains(case, n, gen):
    """q, k, v, g (logarithm of the decay) and beta of n rows: features of unit length as a normalised layer gives them."""
    dtype, hk, hv, dk, dv = DTYPES[case["dtype"]], case["hk"], case["hv"], case["dk"], case["dv"]
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    common = _normal((1, hk, dk), gen)                 # rows of a chain are alike to a degree
    q = unit(_normal((n, hk, dk), gen) + 0.5 * common).to(dtype)
    k = unit(_normal((n, hk, dk), gen) + 0.5 * common).to(dtype)
    v = _normal((n, hv, dv), gen).to(dtype)
    rate = torch.exp(_normal((1, hv), gen) - 3.0)
    g = (-rate * torch.nn.functional.softplus(_normal((n, hv), gen))).to(dtype)
    beta = torch.sigmoid(_normal((n, hv), gen)).to(dtype)
    return q, k, v, g, beta


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)
    op = case["op"]
    s = {"case": case, "op": op, "ctx": None}
    if op in ("dispatch", "combine", "regrad"):
        dtype = DTYPES[case["dtype"]]
        s["node"] = _assign(case, gen)
        places = case["rows"] * case["top"]
        if op == "dispatch":
            s["x"] = _normal((case["rows"], case["d"]), gen).to(dtype)
            s["out"] = torch.zeros(places, case["d"], dtype=dtype, device="cuda")  # rows behind the last node's stay as they are
        else:
            s["y"] = (_normal((places, case["d"]), gen) * torch.exp(0.3 * _normal((places, 1), gen))).to(dtype)
            s["where"], _ = _positions(s["node"])
            s["weights"] = torch.softmax(_normal((case["rows"], case["top"]), gen), 1).contiguous()
            if op == "regrad":
                s["dout"] = _normal((case["rows"], case["d"]), gen).to(dtype)
                s["dy"] = torch.zeros_like(s["y"])
    elif op in ("chain", "chaingrad"):
        s["q"], s["k"], s["v"], s["g"], s["beta"] = _rows_of_chains(case, case["rows"], gen)
        lengths = _lengths(case)
        s["lengths"], s["shard_off"] = lengths, torch.tensor([0] + lengths, device="cuda").cumsum(0)
        s["W0"] = 0.5 * _normal((case["chains"], case["hv"], case["dv"], case["dk"]), gen) if case.get("start") else None
        if op == "chaingrad":
            s["dout"] = _normal(s["v"].shape, gen).to(s["v"].dtype)
    else:
        s["q"], s["k"], s["v"], s["g"], s["beta"] = _rows_of_chains(case, case["chains"], gen)
        s["W"] = 0.5 * _normal((case["pool"], case["hv"], case["dv"], case["dk"]), gen)
        s["slots"] = torch.randperm(case["pool"], generator=gen, device="cuda")[:case["chains"]].to(torch.int32).contiguous()
    if own:
        import paper_1708_04801_b200 as P

        s["ctx"] = P.Context(case.get("nodes", case.get("chains", 1)), case.get("d", case.get("dk", 1)))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------
def _dispatch(s):
    node, nodes = s["node"], s["case"]["nodes"]
    if own:
        where, order, off = s["ctx"].sort_rows(node, nodes)
        return {"where": where, "order": order, "shard_off": off, "rows": s["ctx"].gather_rows(s["x"], where, s["out"])}
    where, order = _positions(node)
    flat = node.reshape(-1)
    kept = (flat >= 0).sum()
    off = torch.searchsorted(torch.where(flat < 0, torch.full_like(flat, nodes), flat)[order].long(), torch.arange(nodes + 1, device=node.device))
    place = torch.arange(order.numel(), device=node.device)
    rows = torch.where((place < kept)[:, None], s["x"][torch.div(order, node.shape[1], rounding_mode="floor")], s["out"])
    return {"where": where, "order": torch.where(place < kept, order, torch.full_like(order, -1)).to(torch.int32), "shard_off": off, "rows": rows}


def _weighted(where, weights):
    return torch.where(where < 0, torch.zeros_like(weights), weights)


def _combine(s):
    if own:
        return s["ctx"].combine_rows(s["y"], s["where"], s["weights"])
    w, at = _weighted(s["where"], s["weights"]), s["where"].clamp_min(0).long()
    out = w[:, :1] * s["y"][at[:, 0]].float()
    for j in range(1, at.shape[1]):
        out = out + w[:, j:j + 1] * s["y"][at[:, j]].float()
    return out.to(s["y"].dtype)


def _regrad(s):
    if own:
        dy, dw = s["ctx"].combine_rows_grad(s["dout"], s["y"], s["where"], s["weights"], s["dy"])
        return {"dy": dy, "dweights": dw}
    dout, at, there = s["dout"].float(), s["where"].clamp_min(0).long(), s["where"] >= 0
    dw = torch.empty_like(s["weights"])
    dy = torch.cat([s["dy"].float(), dout[:1]])  # and a row for what goes nowhere
    for j in range(at.shape[1]):
        dw[:, j] = torch.where(there[:, j], (dout * s["y"][at[:, j]].float()).sum(1), torch.zeros_like(dw[:, j]))
        dy[torch.where(there[:, j], at[:, j], torch.full_like(at[:, j], len(s["y"])))] = s["weights"][:, j:j + 1] * dout
    return {"dy": dy[:-1].to(s["y"].dtype), "dweights": dw}


class _Chunks:
    """The rows of ragged chains as [chains, heads, chunks, CHUNK, ...] in 32 bits, zeros behind each chain's end, and back."""

    def __init__(self, s):
        c, dev = s["case"], s["q"].device
        self.hk, self.hv = c["hk"], c["hv"]
        self.rows = c["rows"]
        longest = max(max(s["lengths"]), 1)
        self.n = -(-longest // CHUNK)
        t = torch.arange(self.n * CHUNK, device=dev)
        off = s["shard_off"]
        self.valid = t[None, :] < (off[1:] - off[:-1])[:, None]
        self.index = torch.where(self.valid, off[:-1, None] + t[None, :], torch.zeros_like(off[:1, None]))

    def split(self, x):
        heads = x.shape[1]
        x = x.float()[self.index] * self.valid.view(*self.valid.shape, *([1] * (x.dim() - 1)))
        x = x.transpose(1, 2)
        if heads != self.hv:
            x = x.repeat_interleave(self.hv // heads, 1)
        return x.reshape(x.shape[0], self.hv, self.n, CHUNK, *x.shape[3:])

    def join(self, x, heads, dtype):
        x = x.reshape(x.shape[0], heads, self.hv // heads, self.n * CHUNK, *x.shape[4:]).sum(2).transpose(1, 2)
        out = torch.zeros(self.rows + 1, *x.shape[2:], device=x.device)  # and a row for what lies behind a chain's end
        out[torch.where(self.valid, self.index, torch.full_like(self.index, self.rows))] = x
        return out[:-1].to(dtype)


def _chain_parts(s):
    """What the chunks need that no model enters: decays, products of rows, and the inverse of a chunk's triangular system."""
    c = _Chunks(s)
    q, k, v = c.split(s["q"]), c.split(s["k"]), c.split(s["v"])
    b = c.split(s["g"]).double().cumsum(-1)           # in 64 bits: differences of sums
    beta = c.split(s["beta"])
    lower = torch.ones(CHUNK, CHUNK, device=q.device).tril()
    D = torch.exp(torch.where(lower > 0, b[..., :, None] - b[..., None, :], torch.full((), -1e4, device=q.device, dtype=torch.float64)).float())
    kk, qk = k @ k.transpose(-1, -2), q @ k.transpose(-1, -2)
    A = beta[..., :, None] * D * kk * lower.tril(-1)
    T = torch.eye(CHUNK, device=q.device).expand_as(A).contiguous()
    for i in range(1, CHUNK):
        T[..., i, :i] = -(A[..., i:i + 1, :i] @ T[..., :i, :i])[..., 0, :]
    return c, q, k, v, beta, b, D, kk, qk * D, T


def _chain_forward(s, parts, keep):
    c, q, k, v, beta, b, D, kk, P, T = parts
    case = s["case"]
    W = torch.zeros(case["chains"], case["hv"], case["dk"], case["dv"], device=q.device) if s["W0"] is None else s["W0"].transpose(-1, -2)
    scale = 1.0 / math.sqrt(case["dk"])
    gamma, rest, last = torch.exp(b).float(), torch.exp(b[..., -1:] - b).float(), torch.exp(b[..., -1]).float()
    o, starts, news = torch.empty_like(v), [], []
    for i in range(c.n):
        U = T[:, :, i] @ (beta[:, :, i, :, None] * (v[:, :, i] - gamma[:, :, i, :, None] * (k[:, :, i] @ W)))
        o[:, :, i] = scale * (gamma[:, :, i, :, None] * (q[:, :, i] @ W) + P[:, :, i] @ U)
        if keep:
            starts.append(W)
            news.append(U)
        W = last[:, :, i, None, None] * W + k[:, :, i].transpose(-1, -2) @ (rest[:, :, i, :, None] * U)
    return o, W, starts, news


def _chain(s):
    if own:
        o, W = s["ctx"].delta_run(s["q"], s["k"], s["v"], s["g"], s["beta"], s["shard_off"], W0=s["W0"])
        return {"out": o, "W": W}
    parts = _chain_parts(s)
    o, W, _, _ = _chain_forward(s, parts, False)
    return {"out": parts[0].join(o, s["case"]["hv"], s["v"].dtype), "W": W.transpose(-1, -2).contiguous()}


def _chaingrad(s):
    if own:
        o, _, saved = s["ctx"].delta_run(s["q"], s["k"], s["v"], s["g"], s["beta"], s["shard_off"], save=True)
        dq, dk, dv, dg, dbeta = s["ctx"].delta_grad(saved, s["dout"])[:5]
        return {"out": o, "dq": dq, "dk": dk, "dv": dv, "dg": dg, "dbeta": dbeta}
    parts = _chain_parts(s)
    c, q, k, v, beta, b, D, kk, P, T = parts
    o, W, starts, news = _chain_forward(s, parts, True)
    case, dtype = s["case"], s["v"].dtype
    do = c.split(s["dout"]) / math.sqrt(case["dk"])
    gamma, rest, last = torch.exp(b).float()[..., None], torch.exp(b[..., -1:] - b).float()[..., None], torch.exp(b[..., -1]).float()[..., None, None]
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dbeta, db = torch.empty_like(beta), torch.empty_like(beta)
    dW = torch.zeros_like(W)
    t = lambda x: x.transpose(-1, -2)  # noqa: E731
    lower = torch.ones(CHUNK, CHUNK, device=q.device).tril()
    for i in range(c.n - 1, -1, -1):
        W0, U, K, Q, B = starts[i], news[i], k[:, :, i], q[:, :, i], beta[:, :, i, :, None]
        ga, re, la, Pi, Di = gamma[:, :, i], rest[:, :, i], last[:, :, i], P[:, :, i], D[:, :, i]
        kW = K @ W0
        dR = t(T[:, :, i]) @ (t(Pi) @ do[:, :, i] + re * (K @ dW))
        dP = do[:, :, i] @ t(U) * lower
        dA = -(dR @ t(U)) * lower.tril(-1)
        E = dA * Di
        toW = ga * (do[:, :, i] @ t(W0))
        Q_side, K_side = (dP * Di) @ K, t(dP * Di) @ Q
        ahead = re * (U @ t(dW))
        x = -ga * (dR @ t(W0)) + E @ K                       # what the row's step itself sends to its features, over beta
        back = K_side + ahead + t(B * E) @ K
        dq[:, :, i] = toW + Q_side
        dk[:, :, i] = B * x + back
        dv[:, :, i] = B * dR
        dbeta[:, :, i] = (dR * v[:, :, i]).sum(-1) + (x * K).sum(-1)
        db[:, :, i] = (Q * dq[:, :, i]).sum(-1) + (K * (B * x - back)).sum(-1)
        db[:, :, i, -1] += (la * W0 * dW).sum((-1, -2)) + (K * ahead).sum((-1, -2))
        dW = la * dW + t(Q * ga) @ do[:, :, i] - t(K * (ga * B)) @ dR
    dg = db.flip(-1).cumsum(-1).flip(-1)
    return {"out": c.join(o, case["hv"], dtype), "dq": c.join(dq, case["hk"], dtype), "dk": c.join(dk, case["hk"], dtype),
            "dv": c.join(dv, case["hv"], dtype), "dg": c.join(dg, case["hv"], dtype), "dbeta": c.join(dbeta, case["hv"], dtype)}


def _step(s):
    if own:
        return {"out": s["ctx"].delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["W"], s["slots"]), "W": s["W"]}
    case, at = s["case"], s["slots"].long()
    more = case["hv"] // case["hk"]
    q, k = s["q"].float().repeat_interleave(more, 1), s["k"].float().repeat_interleave(more, 1)
    W = s["W"][at] * torch.exp(s["g"].float())[..., None, None]
    W = W + (s["beta"].float()[..., None] * (s["v"].float() - (W * k[:, :, None]).sum(-1)))[..., None] * k[:, :, None]
    s["W"][at] = W
    return {"out": ((W * q[:, :, None]).sum(-1) / math.sqrt(case["dk"])).to(s["v"].dtype), "W": s["W"]}


def run(state):
    return {"dispatch": _dispatch, "combine": _combine, "regrad": _regrad, "chain": _chain, "chaingrad": _chaingrad, "step": _step}[state["op"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------
def work(case):
    op, es = case["op"], 4 if case["dtype"] == "f32" else 2
    if op in ("dispatch", "combine", "regrad"):
        rows, top, d = case["rows"], case["top"], case["d"]
        there = rows * top * (0.85 if case["dropped"] else 1.0)
        if op == "dispatch":
            return {"bytes": rows * top * 12 + 8 * case["nodes"] + (rows + there) * d * es, "flops": 0}
        if op == "combine":
            return {"bytes": rows * top * 8 + (rows + there) * d * es, "flops": 2 * there * d}
        return {"bytes": rows * top * 12 + (rows + 2 * there) * d * es, "flops": 3 * there * d}
    hk, hv, dk, dv = case["hk"], case["hv"], case["dk"], case["dv"]
    n = case["chains"] if op == "step" else case["rows"]
    inputs, out, models = n * (2 * hk * dk + hv * dv + 2 * hv) * es, n * hv * dv * es, case["chains"] * hv * dk * dv * 4
    per_row = 7 * n * hv * dk * dv  # decay, margins, step and answers
    if op == "step":
        return {"bytes": inputs + out + 2 * models, "flops": per_row}
    if op == "chain":
        return {"bytes": inputs + out + (2 if case["start"] else 1) * models, "flops": per_row}
    return {"bytes": 2 * inputs + 2 * out, "flops": 3 * per_row}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------
def _rows_in_64(q, k, v, g, beta, W, scale):
    """The recurrence row by row for chains side by side; inputs [chains, heads, ...] per row. Returns the answers and the models."""
    out = []
    for t in range(len(q)):
        W = W * g[t].exp()[..., None, None]
        miss = v[t] - torch.einsum("chvk,chk->chv", W, k[t])
        W = W + torch.einsum("chv,chk->chvk", beta[t][..., None] * miss, k[t])
        out.append(scale * torch.einsum("chvk,chk->chv", W, q[t]))
    return out, W


def exact(case, seed):
    op = case["op"]
    longest = max(_lengths(case)) if op in ("chain", "chaingrad") else 0
    state = case.get("chains", 0) * case.get("hv", 0) * case.get("dk", 0) * case.get("dv", 0)
    if longest * (60e-6 + state * 40 / 2e12) * (1 if op == "chain" else 6) > 15:
        return None
    s = prepare(case, seed)
    if op == "dispatch":
        node = s["node"].reshape(-1).long()
        places = node.numel()
        keys = (node + 1) * places + torch.arange(places, device=node.device)  # all different, padding first
        first = int((node < 0).sum())
        at = keys.sort().values[first:] % places
        rows = s["out"].double()
        rows[:len(at)] = s["x"][at // case["top"]].double()
        return {"where": None, "order": None, "shard_off": None, "rows": rows}
    if op in ("combine", "regrad"):
        place, w = s["where"].cpu(), s["weights"].double()
        y = s["y"]
        sure = torch.where(place < 0, torch.zeros_like(place), place).long().to(y.device)
        kept = (place >= 0).to(y.device)
        if op == "combine":
            total = torch.zeros(case["rows"], case["d"], dtype=torch.float64, device=y.device)
            for at in range(0, case["rows"], 16384):
                part = slice(at, at + 16384)
                total[part] = torch.einsum("rt,rtd->rd", w[part] * kept[part], y[sure[part]].double())
            return total
        dy = s["dy"].double()
        dw = torch.zeros_like(w)
        for at in range(0, case["rows"], 16384):
            part = slice(at, at + 16384)
            dout = s["dout"][part].double()
            dw[part] = torch.einsum("rd,rtd->rt", dout, y[sure[part]].double()) * kept[part]
            r, j = kept[part].nonzero(as_tuple=True)
            dy[sure[part][r, j]] = w[part][r, j, None] * dout[r]
        return {"dy": dy, "dweights": dw}
    more, scale = case["hv"] // case["hk"], case["dk"] ** -0.5
    wide = lambda x: x.double().repeat_interleave(more, 1)  # noqa: E731
    if op == "step":
        at = s["slots"].long()
        models = s["W"].double()
        out, W = _rows_in_64([wide(s["q"])], [wide(s["k"])], [s["v"].double()], [s["g"].double()], [s["beta"].double()], models[at], scale)
        models[at] = W
        return {"out": out[0], "W": models}
    lengths, off = s["lengths"], s["shard_off"].tolist()
    dev = s["q"].device
    longest = max(lengths)
    W = torch.zeros(case["chains"], case["hv"], case["dv"], case["dk"], dtype=torch.float64, device=dev) if s["W0"] is None else s["W0"].double()
    names = ("q", "k", "v", "g", "beta")
    ends, starts = torch.tensor(lengths, device=dev), torch.tensor(off[:-1], device=dev)

    def rows(t0, t1):
        """Rows t0..t1 of every chain, as leaves: steps of nothing behind a chain's end."""
        t = torch.arange(t0, t1, device=dev)[:, None]
        here = t < ends[None]
        index = torch.where(here, starts[None] + t, torch.zeros_like(t))
        got = []
        for name in names:
            x = s[name][index].double()
            got.append(x * here.view(*here.shape, *([1] * (x.dim() - 2))))
        return got, index, here

    def forward(x, W):
        q, k = x[0].repeat_interleave(more, 2), x[1].repeat_interleave(more, 2)
        return _rows_in_64(q.unbind(0), k.unbind(0), x[2].unbind(0), x[3].unbind(0), x[4].unbind(0), W, scale)

    answers = torch.zeros(s["v"].shape, dtype=torch.float64, device=dev)
    span, kept = 32, []
    for t0 in range(0, longest, span):
        if op == "chaingrad":
            kept.append(W)
        x, index, here = rows(t0, min(longest, t0 + span))
        o, W = forward(x, W)
        answers[index[here]] = torch.stack(o)[here]
    if op == "chain":
        return {"out": answers, "W": W}
    grads = [torch.zeros(s[name].shape, dtype=torch.float64, device=dev) for name in names]
    dW = torch.zeros_like(W)
    for i in range(len(kept) - 1, -1, -1):
        t0 = i * span
        x, index, here = rows(t0, min(longest, t0 + span))
        leaves = [y.requires_grad_(True) for y in x] + [kept[i].detach().requires_grad_(True)]
        with torch.enable_grad():
            o, end = forward(leaves[:5], leaves[5])
            dout = s["dout"][index].double() * here[..., None, None]
            value = (torch.stack(o) * dout).sum() + (end * dW).sum()
        got = torch.autograd.grad(value, leaves)
        for total, part in zip(grads, got[:5]):
            total[index[here]] = part[here]
        dW = got[5]
    return {"out": answers, "dq": grads[0], "dk": grads[1], "dv": grads[2], "dg": grads[3], "dbeta": grads[4]}
