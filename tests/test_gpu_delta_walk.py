"""Chains whose heads have more than 64 labels, which walk by tcgen05, at what the other walk is tested at as well (models in place, strides, ends of the gates, NaN, graphs, rows past
32 bits); and how far answers, models and gradients of bf16 chains are from 64 bits, each by a bound of its own.

Bounds of norms. A rounding to bf16 is off by delta 2^-8 / m of a value with mantissa m, delta even in [-1, 1]; over mantissas even in their logarithm the square has the mean 2^-16 / 3 * E[m^-2],
E[m^-2] = 3 / (8 ln 2): RHO = 0.425 * 2^-8 of the norm. Roundings of different operands are independent of each other, so that their squares add up, and a sum of products of a rounded operand is
off by that operand's share at most. Roundings one behind the other: answers 2 (models in S Q^T, the answer); labels 1 (the gradient itself: all before it is split in two parts); queries 3 (U, F,
itself; S instead of U and F on the other way); features 4 (U, dR, E, itself); steps 5 (U, dR, E, D o K K^T, itself); decays 6 (S, G, U, dR, D o K K^T, itself). A tenth above that for the split
products and for chance. Models: three split products of 2^-17 each one behind the other, which the triangular inverse passes on, a factor of 4 as elsewhere: 4 * 3 * 2^-17 is 9.2e-5 at most where
all errors agree; independent signs over the 64 rows of a chunk leave an eighth of that, 2^-16.5 < 1.2e-5."""
import math

import pytest
import torch

from test_gpu_delta import check_run, gen, make, offsets, reference, reference_grad

pytestmark = pytest.mark.gpu

RHO = 0.425 * 2.0 ** -8
ROUNDINGS = {"out": 2, "dq": 3, "dk": 4, "dv": 1, "dg": 6, "dbeta": 5}
MODELS = 1.2e-5


@pytest.fixture(scope="module")
def P(wpsgd_lib):
    import paper_1708_04801_b200 as pkg

    return pkg


@pytest.fixture(scope="module")
def ctx(P):
    with P.Context(4, 8) as c:
        yield c
        c.check()


def off_16(shape, by):
    """A contiguous fp32 tensor that starts `by` elements behind a multiple of 16 bytes."""
    return torch.zeros(math.prod(shape) + 4, device="cuda")[by:by + math.prod(shape)].view(shape)


@pytest.mark.parametrize("by", [0, 1])
@pytest.mark.parametrize("dk,dv", [(48, 72), (128, 128), (33, 97), (64, 65), (126, 88)])
def test_strides_scale_and_models_in_place(ctx, dk, dv, by):
    n, h = 150, 2
    rows = make(n, h, h, dk, dv, torch.bfloat16, 5)
    wide = torch.full((n, 2 * h * dk + h * dv + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    parts, at = [], 0
    for x in rows[:3]:
        w = x.shape[1] * x.shape[2]
        parts.append(wide[:, at:at + w].unflatten(1, x.shape[1:]))
        parts[-1].copy_(x)
        at += w
    gates = torch.full((n, 3 * h + 1), float("nan"), dtype=torch.bfloat16, device="cuda")
    for i, x in enumerate(rows[3:]):
        parts.append(gates[:, 1 + i * h:1 + (i + 1) * h])
        parts[-1].copy_(x)
    to = torch.full((n, h * dv + 5), 3.0, dtype=torch.bfloat16, device="cuda")
    out = to[:, 1:1 + h * dv].unflatten(1, (h, dv))
    off = offsets([100, 50])
    W0 = torch.randn((2, h, dv, dk), generator=gen(1))
    W = off_16(W0.shape, by)
    W.copy_(W0)
    got = ctx.delta_run(*parts, off.cuda(), W0=W, W_out=W, out=out, scale=0.7)
    ctx.check()
    assert got[1] is W and bool((to[:, 0] == 3).all()) and bool((to[:, 1 + h * dv:] == 3).all())
    check_run(rows, off, got, W0, 0.7)
    # the same from models and to models elsewhere
    apart = off_16(W0.shape, 1 - by)
    again = ctx.delta_run(*[x.cuda() for x in rows], off.cuda(), W0=W0.cuda(), W_out=apart, scale=0.7)
    ctx.check()
    assert torch.equal(again[0], out) and torch.equal(apart, W)


@pytest.mark.parametrize("dk,dv", [(32, 96), (128, 128)])
def test_ends_of_the_gates(ctx, dk, dv):
    n = 200
    rows = make(n, 1, 2, dk, dv, torch.bfloat16, 9)
    rows[3][10], rows[3][75], rows[3][76], rows[3][130] = -float("inf"), -500.0, -100.0, -128.0
    rows[3][20:40] = 0.0
    rows[4][30:45] = 0.0
    rows[4][90:110] = 1.0
    off = offsets([n])
    got = ctx.delta_run(*[x.cuda() for x in rows], off.cuda())
    ctx.check()
    check_run(rows, off, got)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nan_stays_in_its_head_and_chain(ctx, bad):
    rows = make(160, 2, 2, 32, 80, torch.bfloat16, 4)
    rows[2][100, 1, 3] = bad
    off = offsets([64, 70, 26])
    out, W = ctx.delta_run(*[x.cuda() for x in rows], off.cuda())
    # row 100 is the 37th of its chain, in the block of 16 from row 96 on: tiles of 16 x 16 multiply it by the zeros that answers before it have for it
    wrong, wrong_out = ~torch.isfinite(W.cpu()), ~torch.isfinite(out.cpu())
    assert bool(wrong[1, 1, 3].all()) and int(wrong.sum()) == 32
    assert bool(wrong_out[100:134, 1, 3].all()) and int(wrong_out.sum()) <= 134 - 96 and int(wrong_out[96:134, 1, 3].sum()) == int(wrong_out.sum())
    ctx.check()


@pytest.mark.parametrize("width,at", [(1 << 20, 0), ((1 << 20) + 1, 3)])
def test_rows_that_lie_past_32_bits(ctx, width, at):
    lengths, hk, hv, dk, dv = [2000, 63, 2041], 2, 4, 64, 128
    n, off = sum(lengths), offsets(lengths).cuda()
    rows = [x.cuda() for x in make(n, hk, hv, dk, dv, torch.bfloat16, 31)]
    wide = torch.empty((n + 1, width), dtype=torch.bfloat16, device="cuda")
    far_rows, c = [], at
    for x in rows + [rows[2], rows[2]]:
        far_rows.append(wide[1:, c:c + x[0].numel()].unflatten(1, x.shape[1:]))
        far_rows[-1].copy_(x)
        c += (x[0].numel() + 7) // 8 * 8
    want = ctx.delta_run(*rows, off, save=True)
    got = ctx.delta_run(*far_rows[:5], off, out=far_rows[5], save=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(torch.equal(a, b) for a, b in zip(ctx.delta_grad(got[2], far_rows[6])[:5], ctx.delta_grad(want[2], rows[2])[:5]))
    ctx.check()


def test_two_graphs(P):
    rows = [[x.cuda() for x in make(330, 1, 2, 128, 128, torch.bfloat16, s)] for s in (1, 2)]
    off = offsets([200, 130]).cuda()
    dout = torch.randn((330, 2, 128), generator=gen(1)).to(torch.bfloat16).cuda()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s), P.Context(2, 64, stream=s) as c:
        want = []
        for r in rows:
            o, W, saved = c.delta_run(*r, off, save=True)
            want.append([x.clone() for x in (o, W) + tuple(c.delta_grad(saved, dout)[:5])])
        graphs, got = [], []
        for r in rows:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                o, W, saved = c.delta_run(*r, off, save=True)
                got.append((o, W) + tuple(c.delta_grad(saved, dout)[:5]))
            graphs.append(graph)
        for _ in range(3):
            for graph in graphs:
                graph.replay()
        s.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
        c.check()
        for graph in graphs:
            graph.reset()


@pytest.mark.parametrize("hk,hv,dk,dv", [(2, 4, 128, 128), (2, 2, 64, 48)])
def test_two_contexts_at_once_and_again(P, hk, hv, dk, dv):
    """The same bits from two streams at once, beside products of packed rows that use tensor memory too, and from call to call."""
    lengths = [700, 64, 1, 300]
    rows = [x.cuda() for x in make(sum(lengths), hk, hv, dk, dv, torch.bfloat16, 8)]
    dout = torch.randn((sum(lengths), hv, dv), generator=gen(1)).to(torch.bfloat16).cuda()
    off = offsets(lengths).cuda()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    x = torch.randn((2000, 256), generator=gen(2)).cuda()
    torch.cuda.synchronize()
    results, products = [], []
    with P.Context(4, 256, stream=streams[0]) as c0, P.Context(4, 256, stream=streams[1]) as c1, P.Context(4, 256, stream=streams[2]) as c2:
        with torch.cuda.stream(streams[2]):
            q, scales = c2.quantize_rows(x)
        for _ in range(8):
            for c, s in zip((c0, c1), streams):
                with torch.cuda.stream(s):
                    o, W, saved = c.delta_run(*rows, off, save=True)
                    results.append((o, W) + tuple(c.delta_grad(saved, dout)[:5]))
            with torch.cuda.stream(streams[2]):
                products.append(c2.margins_fp8(q, scales, q, scales))
        torch.cuda.synchronize()
        for c in (c0, c1, c2):
            c.check()
        assert all(torch.equal(a, b) for r in results for a, b in zip(r, results[0])) and all(torch.equal(z, products[0]) for z in products)


def shares(name, got, want):
    """Errors over their bound: of the whole, and of the worst head and run of 64 rows, a half above the bound of what such a piece and the mean piece have."""
    bound = 1.1 * RHO * ROUNDINGS[name] ** 0.5
    e, w = (x.cpu().double().flatten(2) if x.dim() == 3 else x.cpu().double()[..., None] for x in (got, want))
    e = e - w
    pad = -len(e) % 64
    e, w = (torch.nn.functional.pad(x, (0, 0, 0, 0, 0, pad)).unflatten(0, (-1, 64)).square().sum((1, 3)) for x in (e, w))
    return float((e.sum() / w.sum()).sqrt()) / bound, float((e / (w + w.mean())).max().sqrt()) / (1.5 * bound)


@pytest.mark.parametrize("start", [False, True])
@pytest.mark.parametrize("lengths,hk,hv,dk,dv", [([300, 100], 1, 2, 128, 128), ([200, 190], 2, 2, 64, 96), ([333], 1, 3, 64, 64), ([150, 64, 170], 2, 2, 100, 40), ([256], 2, 2, 128, 16)])
def test_how_far_results_are_from_64_bits(ctx, lengths, hk, hv, dk, dv, start):
    n, off = sum(lengths), offsets(lengths)
    rows = make(n, hk, hv, dk, dv, torch.bfloat16, 41)
    dout = torch.randn((n, hv, dv), generator=gen(4)).to(torch.bfloat16)
    W0, dW = (torch.randn((len(lengths), hv, dv, dk), generator=gen(s)) if start else None for s in (5, 6))
    on = [x.cuda() for x in rows]
    o, W, saved = ctx.delta_run(*on, off.cuda(), W0=None if W0 is None else W0.cuda(), save=True)
    grads = ctx.delta_grad(saved, dout.cuda(), None if dW is None else dW.cuda(), start=True)
    ctx.check()
    want_o, want_W = reference(rows, off, W0)[:2]
    want = reference_grad(rows, off, dout, dW, W0)
    away = {name: shares(name, a, b) for name, a, b in zip(("out", "dq", "dk", "dv", "dg", "dbeta"), (o,) + tuple(grads[:5]), [want_o] + want[:5])}
    for name, a, b in (("W", W, want_W), ("dW0", grads[5], want[5])):
        away[name] = (float((a.cpu().double() - b).norm() / b.norm()) / MODELS,)
    assert all(x <= 1 for v in away.values() for x in v), away


# ---- rows by node for the chains of one label a row ------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_sorted_by_node_are_what_run_takes(P, dtype):
    """sort_rows and gather_rows lay rows and labels out for run, whose offsets are on the host; the same rows sorted on the host give the same models."""
    n, k, d = 500, 6, 96
    x = torch.randn((n, d), generator=gen(1)).to(dtype)
    y = torch.randint(0, 2, (n,), generator=gen(2)).float() * 2 - 1
    node = torch.randint(0, k, (n, 1), generator=gen(3), dtype=torch.int32)
    node[::11] = -1
    with P.Context(k, d) as c:
        where, _, off = c.sort_rows(node.cuda())
        X, Y = c.gather_rows(x.cuda(), where), c.gather_rows(y[:, None].cuda(), where)
        steps = [50 + 10 * j for j in range(k)]
        c.run(X, Y.view(-1), off.cpu(), steps, 0.05, P.LR_CONST, 0.01, P.LOSS_LOGISTIC, 7)
        got = c.combine()
        order = torch.argsort(node.view(-1), stable=True)
        order = order[node.view(-1)[order] >= 0]
        c.run(x[order].cuda(), y[order].cuda(), off.cpu(), steps, 0.05, P.LR_CONST, 0.01, P.LOSS_LOGISTIC, 7)
        assert torch.equal(got, c.combine()) and bool(got.any())
        c.check()
