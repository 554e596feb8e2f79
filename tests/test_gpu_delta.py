"""Chains whose labels are vectors (gated delta rule), through the public entry points, against the recurrence row by row in 64 bits.

Tolerances. Let A be the models' recurrence with the sizes of all terms, A <- e^g A + beta (|v| + |W| |k|) |k|^T: a step beta (v - W k) is a difference, so what its
roundings leave goes by the sizes of v and of the products in W k and not by the step. scale A |q| has those of the answers. fp32 rows: a row has at most dk + 8 roundings of u = 2^-24 in each sum, and errors of earlier rows are carried
on by a contraction. bf16 rows on the tensor cores: operands on the fp32 side are split in two parts that leave 2^-17 of them; three products follow each other in a chunk,
and the triangular inverse passes errors on, counted as a factor of 4: 4 * 3 * 2^-17 < 2^-13 of A. Answers take products of the chunk and old models
rounded to bf16 once (half a step is 2^-8), and are rounded once themselves."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def P(wpsgd_lib):
    import paper_1708_04801_b200 as pkg

    return pkg


@pytest.fixture(scope="module")
def ctx(P):
    with P.Context(4, 8) as c:
        yield c
        c.check()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make(n, hk, hv, dk, dv, dtype, seed=0, unit=True):
    g = gen(1000 * seed + n)
    q, k, v = (torch.randn(s, generator=g) for s in ((n, hk, dk), (n, hk, dk), (n, hv, dv)))
    if unit:
        q, k = (x / x.norm(dim=-1, keepdim=True).clamp_min(1e-6) for x in (q + 0.3, k + 0.3))
    decay = -torch.exp(torch.randn((n, hv), generator=g) - 2.0)
    beta = torch.sigmoid(torch.randn((n, hv), generator=g))
    return [x.to(dtype) for x in (q, k, v, decay, beta)]


def offsets(lengths, first=0):
    return torch.tensor([first] + lengths).cumsum(0)


def reference(rows, off, W0=None, scale=None):
    """(out, W, sizes of out, sizes of W) in 64 bits, row by row; rows outside the chains are zeros in out."""
    q, k, v, g, beta = (x.double().cpu() for x in rows)
    hv, more = v.shape[1], v.shape[1] // q.shape[1]
    q, k = q.repeat_interleave(more, 1), k.repeat_interleave(more, 1)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    chains = len(off) - 1
    out, size = torch.zeros_like(v), torch.zeros_like(v)
    W_all = torch.zeros(chains, hv, v.shape[2], q.shape[2], dtype=torch.float64) if W0 is None else W0.double().cpu().clone()
    A_all = W_all.abs()
    for c in range(chains):
        W, A = W_all[c], A_all[c]
        for t in range(int(off[c]), int(off[c + 1])):
            a = torch.exp(g[t])[:, None, None]
            W = a * W
            step = beta[t][:, None] * (v[t] - torch.einsum("hvk,hk->hv", W, k[t]))
            sized = beta[t][:, None] * (v[t].abs() + torch.einsum("hvk,hk->hv", W.abs(), k[t].abs()))
            W = W + step[..., None] * k[t][:, None]
            A = a * A + sized[..., None] * k[t].abs()[:, None]
            out[t] = scale * torch.einsum("hvk,hk->hv", W, q[t])
            size[t] = abs(scale) * torch.einsum("hvk,hk->hv", A, q[t].abs())
        W_all[c], A_all[c] = W, A
    return out, W_all, size, A_all


def within(error, bound):
    """The largest error over its bound."""
    return float((error.abs() / (bound + 1e-30)).max()) if error.numel() else 0.0


def check_run(rows, off, got, W0=None, scale=None, exact_rows=None):
    out, W = got[0].cpu().double(), got[1].cpu().double()
    want, models, size, A = reference(rows, off, W0, scale)
    dtype, dk = rows[0].dtype, rows[0].shape[2]
    longest = max(int(off[i + 1] - off[i]) for i in range(len(off) - 1)) if len(off) > 1 else 0
    if dtype is torch.float32 or exact_rows:
        # a row's error, (dk + 8) u of the sizes; those of earlier rows fade with the contraction, at worst they add up
        part = (dk + 8) * U * (4 + longest ** 0.5)
        bound_w, bound_o = part * A, part * size + HALF[dtype] * want.abs()
    else:
        bound_w, bound_o = 2.0 ** -13 * A, 2.0 ** -8 * (2 * size + want.abs()) * 1.02
    inside = torch.zeros(len(want), dtype=torch.bool)
    inside[int(off[0]):int(off[-1])] = True
    far_o, far_w = within((out - want)[inside], bound_o[inside]), within(W - models, bound_w)
    assert far_o <= 1 and far_w <= 1


CASES = [  # lengths, first row, rows behind, heads_k, heads_v, dk, dv
    ([1], 0, 0, 1, 1, 1, 1), ([0, 3, 0], 0, 2, 1, 1, 5, 3), ([7, 1, 64], 3, 5, 2, 2, 16, 16), ([65, 63, 64, 0], 0, 0, 1, 2, 64, 64), ([130], 1, 0, 2, 6, 128, 128),
    ([33, 100, 200], 0, 1, 3, 3, 60, 33), ([257, 5], 0, 0, 1, 3, 97, 128), ([90], 0, 0, 2, 2, 128, 17), ([300], 0, 7, 1, 1, 32, 8), ([64, 128], 0, 0, 1, 1, 72, 40),
    ([65, 0, 200], 2, 3, 1, 2, 40, 128), ([64, 129], 0, 0, 2, 2, 64, 65), ([1, 320], 0, 1, 1, 1, 128, 81),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("start", [False, True])
@pytest.mark.parametrize("lengths,first,behind,hk,hv,dk,dv", CASES)
def test_run(ctx, lengths, first, behind, hk, hv, dk, dv, start, dtype):
    n = first + sum(lengths) + behind
    rows = make(n, hk, hv, dk, dv, dtype, dk)
    off = offsets(lengths, first)
    W0 = torch.randn((len(lengths), hv, dv, dk), generator=gen(3)) if start else None
    on = [x.cuda() for x in rows]
    for x in on:  # rows outside the chains are not read
        x[:first] = float("nan")
        x[n - behind:] = float("nan")
    out = torch.full((n, hv, dv), 7.0, dtype=dtype, device="cuda")
    got = ctx.delta_run(*on, off.cuda(), W0=None if W0 is None else W0.cuda(), out=out)
    ctx.check()
    assert got[0] is out and bool((out[:first] == 7).all()) and bool((out[n - behind:] == 7).all())
    check_run(rows, off, got, W0)


# what the library chooses from: labels as lanes of tensor memory or shared by 8, 4 or 2 warps of a block, heads that share features formed together, rows by tensor maps or not, rings that go round
FORMS = [([260, 200, 130, 64] * 10, 2, 4, 128, 128), ([260, 200, 130, 64] * 10, 4, 4, 64, 64), ([3] * 600, 4, 8, 128, 128), ([1, 65] * 150, 2, 6, 64, 64), ([2] * 400, 4, 12, 24, 32),
         ([70] * 80, 2, 2, 72, 120), ([200, 3] * 80, 1, 1, 128, 72), ([200, 3] * 80, 1, 2, 64, 128), ([150, 64] * 40, 2, 2, 24, 100)]


@pytest.mark.parametrize("lengths,hk,hv,dk,dv", FORMS)
def test_run_forms(ctx, lengths, hk, hv, dk, dv):
    rows = make(sum(lengths), hk, hv, dk, dv, torch.bfloat16, 21)
    off = offsets(lengths)
    W0 = torch.randn((len(lengths), hv, dv, dk), generator=gen(3))
    on = [x.cuda() for x in rows]
    got = ctx.delta_run(*on, off.cuda(), W0=W0.cuda())
    ctx.check()
    out, W = got
    # row by row in fp32, which has tests of its own against 64 bits, stands for the recurrence; sizes from there too
    exact_out, exact_W = ctx.delta_run(*[x.float() for x in on], off.cuda(), W0=W0.cuda())
    sized_out, sized_W = ctx.delta_run(on[0].float().abs(), on[1].float().abs(), 3 * on[2].float().abs(), on[3].float(), on[4].float(), off.cuda(), W0=W0.abs().cuda())
    ctx.check()
    assert float((W - exact_W).norm()) <= 2.0 ** -13 * float(exact_W.norm() + sized_W.norm())
    assert float((out.float() - exact_out).norm()) <= 3 * 2.0 ** -8 * float(exact_out.norm())


@pytest.mark.parametrize("lengths,hk,hv,dk,dv", FORMS)
def test_gradients_forms(ctx, lengths, hk, hv, dk, dv):
    """Gradients of many chains at once are, bit for bit, those of the chains a few at a time, which other tests hold against 64 bits."""
    n = sum(lengths)
    rows = [x.cuda() for x in make(n, hk, hv, dk, dv, torch.bfloat16, 22)]
    dout = torch.randn((n, hv, dv), generator=gen(4)).to(torch.bfloat16).cuda()
    off = offsets(lengths)
    out, W, saved = ctx.delta_run(*rows, off.cuda(), save=True)
    got = ctx.delta_grad(saved, dout)[:5]
    for a, b in ((0, 1), (len(lengths) - 2, len(lengths))):
        part = slice(int(off[a]), int(off[b]))
        few = [x[part].contiguous() for x in rows]
        o, w, kept = ctx.delta_run(*few, (off[a:b + 1] - off[a]).cuda(), save=True)
        same = [torch.equal(x[part], y) for x, y in zip(got, ctx.delta_grad(kept, dout[part].contiguous())[:5])]
        assert torch.equal(out[part], o) and torch.equal(W[a:b], w) and all(same), same
    ctx.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nothing_to_run(ctx, dtype):
    rows = [x.cuda() for x in make(5, 1, 2, 16, 8, dtype)]
    W0 = torch.randn((3, 2, 8, 16), generator=gen(1)).cuda()
    out = torch.full((5, 2, 8), 7.0, dtype=dtype, device="cuda")
    _, W = ctx.delta_run(*rows, torch.tensor([2, 2, 2, 2]).cuda(), W0=W0, out=out)             # chains without rows keep their models
    assert torch.equal(W, W0) and bool((out == 7).all())
    _, W = ctx.delta_run(*[x[:0] for x in rows], torch.tensor([0, 0]).cuda())                      # no rows at all
    assert W.shape == (1, 2, 8, 16) and float(W.abs().max()) == 0.0
    o, W = ctx.delta_run(*rows, torch.tensor([0]).cuda(), out=out)                              # no chains
    assert W.shape[0] == 0 and bool((o == 7).all())
    ctx.delta_step(*[x[:0] for x in rows], W0)
    if dtype is torch.bfloat16:
        _, _, saved = ctx.delta_run(*rows, torch.tensor([2, 2, 2, 2]).cuda(), save=True)
        dW = torch.randn((3, 2, 8, 16), generator=gen(2)).cuda()
        assert torch.equal(ctx.delta_grad(saved, rows[2], dW, start=True)[5], dW)
    ctx.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_run_strides_scale_and_models_in_place(ctx, dtype):
    # q, k and v of one wide row, as one projection leaves them; answers into part of wider rows; models updated where they are
    n, h, dk, dv = 150, 2, 48, 24
    rows = make(n, h, h, dk, dv, dtype, 5)
    wide = torch.full((n, 2 * h * dk + h * dv + 8), float("nan"), dtype=dtype, device="cuda")
    parts, at = [], 0
    for x in rows[:3]:
        w = x.shape[1] * x.shape[2]
        parts.append(wide[:, at:at + w].unflatten(1, x.shape[1:]))
        parts[-1].copy_(x)
        at += w
    gates = torch.full((n, 3 * h + 1), float("nan"), dtype=dtype, device="cuda")
    for i, x in enumerate(rows[3:]):
        parts.append(gates[:, 1 + i * h:1 + (i + 1) * h])
        parts[-1].copy_(x)
    to = torch.full((n, h * dv + 5), 3.0, dtype=dtype, device="cuda")
    out = to[:, 1:1 + h * dv].unflatten(1, (h, dv))
    off = offsets([100, 50])
    W0 = torch.randn((2, h, dv, dk), generator=gen(1))
    W = W0.cuda()
    got = ctx.delta_run(*parts, off.cuda(), W0=W, W_out=W, out=out, scale=0.7)
    ctx.check()
    assert got[1] is W and bool((to[:, 0] == 3).all()) and bool((to[:, 1 + h * dv:] == 3).all())
    check_run(rows, off, got, W0, 0.7)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_run_at_the_ends_of_the_gates(ctx, dtype):
    # decays that forget everything (also minus infinity), steps of zero (rows that only decay), of one, and decays of one
    n = 200
    rows = make(n, 1, 2, 32, 16, dtype, 9)
    rows[3][10], rows[3][75], rows[3][76], rows[3][130] = -float("inf"), -500.0, -100.0, -128.0
    rows[3][20:40] = 0.0
    rows[4][30:45] = 0.0
    rows[4][90:110] = 1.0
    off = offsets([n])
    got = ctx.delta_run(*[x.cuda() for x in rows], off.cuda())
    ctx.check()
    check_run(rows, off, got)


def test_nan_stays_in_its_head_and_chain(ctx):
    rows = make(160, 2, 2, 32, 16, torch.bfloat16, 4)
    rows[2][100, 1, 3] = float("nan")
    off = offsets([64, 70, 26])
    out, W = ctx.delta_run(*[x.cuda() for x in rows], off.cuda())
    # row 100 is the 37th of its chain, in the block of 16 from row 96 on: tiles of 16 x 16 multiply it by the zeros that answers before it have for it
    bad, bad_out = torch.isnan(W.cpu()), torch.isnan(out.cpu())
    assert bool(bad[1, 1, 3].all()) and int(bad.sum()) == 32
    assert bool(bad_out[100:134, 1, 3].all()) and int(bad_out.sum()) <= 134 - 96 and int(bad_out[96:134, 1, 3].sum()) == int(bad_out.sum())
    ctx.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_bad_offsets_are_reported(P, dtype):
    rows = [x.cuda() for x in make(50, 1, 1, 16, 16, dtype)]
    for off in ([0, 30, 20], [0, 51], [-1, 20], [0, 1 << 40]):
        with P.Context(1, 1) as c:
            c.delta_run(*rows, torch.tensor(off).cuda())
            with pytest.raises(P.WpsgdError):
                c.check()


# ---- gradients ---------------------------------------------------------------------------------------------------------------
def reference_grad(rows, off, dout, dW=None, W0=None, scale=None):
    """Gradients of sum(out dout) + sum(W dW), by automatic differentiation of the recurrence in 64 bits: [dq, dk, dv, dg, dbeta, dW0]."""
    leaves = [x.double().cpu().requires_grad_(True) for x in rows]
    q, k, v, g, beta = leaves
    hv, more = v.shape[1], v.shape[1] // q.shape[1]
    chains = len(off) - 1
    first = (torch.zeros(chains, hv, v.shape[2], q.shape[2], dtype=torch.float64) if W0 is None else W0.double()).requires_grad_(True)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    qq, kk = q.repeat_interleave(more, 1), k.repeat_interleave(more, 1)
    total = torch.zeros((), dtype=torch.float64)
    for c in range(chains):
        W = first[c]
        for t in range(int(off[c]), int(off[c + 1])):
            W = torch.exp(g[t])[:, None, None] * W
            W = W + (beta[t][:, None] * (v[t] - torch.einsum("hvk,hk->hv", W, kk[t])))[..., None] * kk[t][:, None]
            total = total + scale * (torch.einsum("hvk,hk->hv", W, qq[t]) * dout[t].double()).sum()
        if dW is not None:
            total = total + (W * dW[c].double()).sum()
    total.backward()
    return [x.grad if x.grad is not None else torch.zeros_like(x) for x in leaves + [first]]


# A gradient is rounded at the end, and on the way to it come, one after the other, at most: P in dU, dR or U as they are kept, E or F. Each is off by
# 2^-8 of its size at most; all four together by 2^-6 of the norm of what they make up, with the split products' share far below.
GRAD_NORM = 2.0 ** -6


def far(got, want):
    """Norm of the difference over that of the result."""
    return float((got.cpu().double() - want).norm() / want.norm().clamp_min(1e-30))


@pytest.mark.parametrize("start", [False, True])
@pytest.mark.parametrize("lengths,first,behind,hk,hv,dk,dv", CASES)
def test_gradients(ctx, lengths, first, behind, hk, hv, dk, dv, start):
    n = first + sum(lengths) + behind
    rows = make(n, hk, hv, dk, dv, torch.bfloat16, dk + 1)
    off = offsets(lengths, first)
    dout = torch.randn((n, hv, dv), generator=gen(4)).to(torch.bfloat16)
    W0, dW = (torch.randn((len(lengths), hv, dv, dk), generator=gen(s)) if start else None for s in (5, 6))
    on = [x.cuda() for x in rows]
    dout_on = dout.cuda()
    for x in on + [dout_on]:
        x[:first] = float("nan")
        x[n - behind:] = float("nan")
    o, W, saved = ctx.delta_run(*on, off.cuda(), W0=None if W0 is None else W0.cuda(), save=True)
    got = ctx.delta_grad(saved, dout_on, None if dW is None else dW.cuda(), start=start)
    ctx.check()
    plain = ctx.delta_run(*on, off.cuda(), W0=None if W0 is None else W0.cuda())
    inside = slice(first, n - behind)
    assert torch.equal(plain[0][inside], o[inside]) and torch.equal(plain[1], W)   # keeping what the gradient needs changes nothing
    want = reference_grad(rows, off, dout, dW, W0)
    inside = slice(first, n - behind)
    away = {name: far(a[inside], b[inside]) for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta"), got, want)}
    assert (got[5] is not None) == start
    if start:
        away["dW0"] = far(got[5], want[5])
    if n == 1 and not start:  # one row from nothing: nothing to decay, an exact zero
        assert float(want[3].abs().max()) == 0.0 and float(got[3].abs().max()) == 0.0
        away.pop("dg")
    assert all(v <= GRAD_NORM for v in away.values()), away


def test_gradients_are_those_of_differences(ctx):
    # along a direction in all inputs at once: (L(x + h e) - L(x - h e)) / 2h with L from the recurrence in 64 bits, at inputs that are bf16 numbers
    rows = make(100, 1, 2, 24, 16, torch.bfloat16, 11)
    off = offsets([70, 30])
    dout = torch.randn((100, 2, 16), generator=gen(1)).to(torch.bfloat16)
    _, _, saved = ctx.delta_run(*[x.cuda() for x in rows], off.cuda(), save=True)
    got = ctx.delta_grad(saved, dout.cuda())
    ctx.check()
    for i in range(5):
        e = torch.randn(rows[i].shape, generator=gen(20 + i)).double()
        h = 1e-5
        value = lambda s: float((reference([x.double() + (s * h * e if j == i else 0) for j, x in enumerate(rows)], off)[0] * dout.double()).sum())  # noqa: E731
        slope = (value(1) - value(-1)) / (2 * h)
        along = float((got[i].cpu().double() * e).sum())
        # the error is 2^-6 of the gradient's norm at most, and lies along e with the norm of a unit vector's share: 4 standard deviations
        assert abs(slope - along) <= 4 * GRAD_NORM * float(got[i].double().norm()) + 1e-6 * abs(slope)


def test_gradients_of_strided_rows_and_at_the_ends_of_the_gates(ctx):
    n = 200
    rows = make(n, 1, 2, 32, 16, torch.bfloat16, 9)
    rows[3][10], rows[3][75], rows[3][130] = -500.0, -100.0, -128.0
    rows[3][20:40] = 0.0
    rows[4][30:45] = 0.0
    rows[4][90:110] = 1.0
    wide = [torch.zeros(n, x[0].numel() + 3, dtype=torch.bfloat16, device="cuda")[:, 1:1 + x[0].numel()].unflatten(1, x.shape[1:]) if x.dim() == 3 else x.cuda() for x in rows]
    for w, x in zip(wide, rows):
        w.copy_(x)
    off = offsets([n])
    dout = torch.randn((n, 2, 16), generator=gen(1)).to(torch.bfloat16)
    dwide = torch.zeros(n, 40, dtype=torch.bfloat16, device="cuda")[:, 8:].unflatten(1, (2, 16))
    dwide.copy_(dout)
    _, _, saved = ctx.delta_run(*wide, off.cuda(), save=True, scale=0.3)
    got = ctx.delta_grad(saved, dwide)
    ctx.check()
    want = reference_grad(rows, off, dout, scale=0.3)
    away = {name: far(a, b) for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta"), got, want)}
    assert all(v <= GRAD_NORM for v in away.values()), away


@pytest.mark.parametrize("dtype,width,at", [(torch.bfloat16, 1 << 20, 0), (torch.bfloat16, (1 << 20) + 1, 3), (torch.float32, 1 << 19, 0)])
def test_rows_that_lie_past_32_bits(ctx, dtype, width, at):
    # slices of one tensor of 2^31 elements and more; the same rows one behind the other give the same bits
    lengths, hk, hv, dk, dv = [2000, 63, 2041], 2, 4, 128, 64
    n, off = sum(lengths), offsets(lengths).cuda()
    rows = [x.cuda() for x in make(n, hk, hv, dk, dv, dtype, 31)]
    wide = torch.empty((n + 1, width), dtype=dtype, device="cuda")
    far_rows, c = [], at
    for x in rows + [rows[2], rows[2]]:  # and places for the answers and their gradient
        far_rows.append(wide[1:, c:c + x[0].numel()].unflatten(1, x.shape[1:]))
        far_rows[-1].copy_(x)
        c += (x[0].numel() + 7) // 8 * 8
    save = dtype is torch.bfloat16
    want = ctx.delta_run(*rows, off, save=save)
    got = ctx.delta_run(*far_rows[:5], off, out=far_rows[5], save=save)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    if save:
        assert all(torch.equal(a, b) for a, b in zip(ctx.delta_grad(got[2], far_rows[6])[:5], ctx.delta_grad(want[2], rows[2])[:5]))
    ctx.check()


def test_workspaces_and_models_past_32_bits(ctx):
    lengths, hk, hv, dk, dv = [4000] * 104 + [77, 4003], 2, 16, 128, 128
    n, off = sum(lengths), offsets(lengths)
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v, gate, beta, dout = (torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16) for s in ((n, hk, dk), (n, hk, dk), (n, hv, dv), (n, hv), (n, hv), (n, hv, dv)))
    rows = [q / 11, k / 11, v, -gate.abs(), torch.sigmoid(beta)]
    out, W, saved = ctx.delta_run(*rows, off.cuda(), save=True)
    assert saved.args[-1].numel() > 1 << 32
    got = ctx.delta_grad(saved, dout)[:5]
    a, b = len(lengths) - 2, len(lengths)
    part = slice(int(off[a]), int(off[b]))
    few = [x[part].contiguous() for x in rows]
    o, w, kept = ctx.delta_run(*few, (off[a:b + 1] - off[a]).cuda(), save=True)
    assert torch.equal(out[part], o) and torch.equal(W[a:b], w)
    assert all(torch.equal(x[part], y) for x, y in zip(got, ctx.delta_grad(kept, dout[part].contiguous())[:5]))
    # single rows on models of which the last lie past 2^31 elements
    del saved, got
    slots = (1 << 31) // (hv * dv * dk) + 5
    pool = torch.zeros((slots, hv, dv, dk), device="cuda")
    pool[-2:] = w
    one = [x[-2:].contiguous() for x in rows]
    mine = w.clone()
    want = ctx.delta_step(*one, mine)
    answer = ctx.delta_step(*one, pool, torch.tensor([slots - 2, slots - 1], dtype=torch.int32).cuda())
    ctx.check()
    assert torch.equal(answer, want) and torch.equal(pool[-2:], mine) and float(pool[:-2].abs().max()) == 0.0


# ---- all of it together ------------------------------------------------------------------------------------------------------------
def test_rows_to_chains_and_back_with_gradients(ctx):
    """A router's rows sorted by chain, run through them, brought back with weights, and the gradients all the way to the inputs."""
    n, top, chains, h, dk, dv = 150, 2, 5, 2, 32, 16
    g = gen(3)
    rows = make(n, h, h, dk, dv, torch.bfloat16, 13)
    node = torch.stack([torch.randperm(chains, generator=g)[:top] for _ in range(n)]).to(torch.int32)
    node[::9, 1] = -1
    weights = torch.softmax(torch.randn((n, top), generator=g), 1)
    dy = torch.randn((n, h * dv), generator=g).to(torch.bfloat16)

    where, order, off = ctx.sort_rows(node.cuda(), chains)
    places = n * top
    laid = [ctx.gather_rows(x.flatten(1).cuda(), where, torch.zeros(places, x[0].numel(), dtype=x.dtype, device="cuda")).unflatten(1, x.shape[1:]) for x in rows]
    out, _, saved = ctx.delta_run(*laid, off, save=True)
    y = ctx.combine_rows(out.flatten(1), where, weights.cuda())
    dout, dweights = ctx.combine_rows_grad(dy.cuda(), out.flatten(1), where, weights.cuda(), torch.zeros(places, h * dv, dtype=torch.bfloat16, device="cuda"))
    grads = ctx.delta_grad(saved, dout.unflatten(1, (h, dv)))[:5]
    back = [ctx.combine_rows(x.flatten(1), where) for x in grads]
    ctx.check()

    leaves = [x.double().requires_grad_(True) for x in rows]
    w = weights.double().requires_grad_(True)
    total, answers = torch.zeros((), dtype=torch.float64), torch.zeros(n, h, dv, dtype=torch.float64)
    for c in range(chains):
        W = torch.zeros(h, dv, dk, dtype=torch.float64)
        for i, j in (node == c).nonzero().tolist():
            q, k, v, lg, be = (x[i] for x in leaves)
            W = torch.exp(lg)[:, None, None] * W
            W = W + (be[:, None] * (v - torch.einsum("hvk,hk->hv", W, k)))[..., None] * k[:, None]
            o = dk ** -0.5 * torch.einsum("hvk,hk->hv", W, q)
            answers[i] += (w[i, j] * o).detach()
            total = total + w[i, j] * (o * dy[i].view(h, dv).double()).sum()
    total.backward()
    # a rounding of the answers and one of the sum; the gradients as above, from gradients rounded once, and rounded once more
    assert far(y, answers.flatten(1)) <= 3 * 2.0 ** -8
    there = node >= 0
    assert far(dweights[there.cuda()], w.grad[there]) <= 3 * 2.0 ** -8
    away = [far(a, x.grad.flatten(1)) for a, x in zip(back, leaves)]
    assert all(v <= GRAD_NORM + 2 * 2.0 ** -8 for v in away), away


def test_two_graphs_and_another_stream(P):
    """Captured runs, gradients and steps share nothing but what the caller shares: two graphs of one context, replayed in turn."""
    rows = [[x.cuda() for x in make(130, 1, 2, 64, 32, torch.bfloat16, s)] for s in (1, 2)]
    off = offsets([100, 30]).cuda()
    dout = torch.randn((130, 2, 32), generator=gen(1)).to(torch.bfloat16).cuda()
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
        for _ in range(2):
            for graph in graphs:
                graph.replay()
        s.synchronize()
        same = [torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y)]
        assert all(same)
        c.check()
        for graph in graphs:
            graph.reset()


@pytest.mark.parametrize("limit", [1, 4096])
@pytest.mark.parametrize("chains,dv", [(1, 64), (160, 64), (160, 128), (2, 128)])  # warps that only copy beside those that multiply, warps that do both, tcgen05
def test_a_wait_that_runs_out_is_reported(P, limit, chains, dv):
    rows = [x.cuda() for x in make(400 * chains, 1, 1, 64, dv, torch.bfloat16)]
    off = offsets([400] * chains).cuda()
    with P.Context(1, 1) as c:
        want, _, saved = c.delta_run(*rows, off, save=True)
        c.check()
        for call in (lambda: c.delta_run(*rows, off), lambda: c.delta_grad(saved, rows[2])):
            c.set_option("test_drop_block", 5)
            c.set_option("spin_limit", limit)
            call()
            with pytest.raises(P.WpsgdError) as e:
                c.check()
            assert e.value.status_name == "TIMEOUT"
        c.set_option("test_drop_block", -1)
        c.set_option("spin_limit", 1 << 20)
        assert torch.equal(c.delta_run(*rows, off)[0], want)   # and the context goes on
        c.check()


# ---- single rows -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,pool,hk,hv,dk,dv", [(1, 1, 1, 1, 1, 1), (4, 6, 4, 4, 64, 64), (3, 3, 2, 6, 97, 33), (70, 70, 1, 2, 128, 128), (9, 20, 3, 3, 30, 5), (300, 310, 2, 2, 16, 16), (40, 41, 8, 16, 100, 128)])
def test_step(ctx, dtype, n, pool, hk, hv, dk, dv):
    rows = make(n, hk, hv, dk, dv, dtype, 2)
    W0 = torch.randn((pool, hv, dv, dk), generator=gen(1))
    slots = torch.randperm(pool, generator=gen(2))[:n].to(torch.int32)
    slots[n // 2] = -1
    W = W0.cuda()
    out = torch.full((n, hv, dv), 7.0, dtype=dtype, device="cuda")
    ctx.delta_step(*[x.cuda() for x in rows], W, slots.cuda(), out=out)
    ctx.check()
    keep = slots >= 0
    want, models, size, A = reference([x[keep] for x in rows], list(range(int(keep.sum()) + 1)), W0[slots[keep].long()])
    # one row: dk + 8 roundings in each sum, one of the answer
    far_o = within(out.cpu().double()[keep] - want, (dk + 8) * U * size + HALF[dtype] * want.abs() * 1.01)
    far_w = within(W.cpu().double()[slots[keep].long()] - models, (dk + 8) * U * A)
    assert far_o <= 1 and far_w <= 1
    assert bool((out[n // 2] == 7).all())
    rest = torch.ones(pool, dtype=torch.bool)
    rest[slots[keep].long()] = False
    assert torch.equal(W.cpu()[rest], W0[rest])


def test_step_without_slots_row_by_row_is_a_run(ctx):
    # fp32: single rows do what a run of the same rows does, bit for bit
    n, chains = 5, 3
    rows = make(n * chains, 2, 2, 40, 24, torch.float32, 6)
    out, W = ctx.delta_run(*[x.cuda() for x in rows], offsets([n] * chains).cuda())
    V = torch.zeros_like(W)
    for t in range(n):
        o = ctx.delta_step(*[x.view(chains, n, *x.shape[1:])[:, t].contiguous().cuda() for x in rows], V)
        assert torch.equal(o, out.view(chains, n, 2, 24)[:, t])
    assert torch.equal(V, W)
    ctx.check()


def test_step_slots_twice_or_past_the_end(P):
    rows = [x.cuda() for x in make(600, 1, 1, 32, 32, torch.float32)]
    W0 = torch.randn((700, 1, 32, 32), generator=gen(1)).cuda()
    slots = torch.arange(600, dtype=torch.int32).cuda()
    with P.Context(1, 1) as c:
        W1 = W0.clone()
        o1 = c.delta_step(*rows, W1, slots)
        c.check()
        slots[5], slots[599], slots[300] = 700, 17, 17     # past the end; one that row 17 has, twice
        W2, out = W0.clone(), torch.full_like(o1, 7.0)
        c.delta_step(*rows, W2, slots, out=out)
        left = torch.zeros(600, dtype=torch.bool)
        left[[5, 300, 599]] = True
        assert bool((out[left] == 7).all()) and torch.equal(out[~left], o1[~left])
        assert torch.equal(W2[:600][~left], W1[:600][~left]) and torch.equal(W2[:600][left], W0[:600][left])
        with pytest.raises(P.WpsgdError):
            c.check()


def test_refusals(P, ctx):
    n = 6
    rows = [x.cuda() for x in make(n, 1, 2, 16, 8, torch.float32)]
    q, k, v, g, b = rows
    off = offsets([n]).cuda()
    W = torch.zeros(n, 2, 8, 16).cuda()
    for call in (lambda: ctx.delta_run(q.half(), k, v, g, b, off), lambda: ctx.delta_run(q, k.bfloat16(), v, g, b, off), lambda: ctx.delta_run(q, k, v, g, b, off.int()),
                 lambda: ctx.delta_run(q, k, v, g, b, off.cpu()), lambda: ctx.delta_step(*rows, W.double()), lambda: ctx.delta_step(*rows, W, off), lambda: ctx.delta_step(*rows, None)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ctx.delta_run(q[:3], k, v, g, b, off), lambda: ctx.delta_run(q, k, v[:, :, ::2], g, b, off), lambda: ctx.delta_run(q, k, v.flip(1)[:, :1], g, b, off),
                 lambda: ctx.delta_run(q, k, v, g, b, off, W0=W), lambda: ctx.delta_run(q, k, v, g, b, off, out=v[:3]), lambda: ctx.delta_step(*rows, W[:, :1].contiguous()),
                 lambda: ctx.delta_step(*rows, W, torch.zeros(2, dtype=torch.int32).cuda())):
        with pytest.raises(ValueError):
            call()
    wide = [x.cuda() for x in make(n, 1, 1, 129, 8, torch.float32)]
    tall = [x.cuda() for x in make(n, 1, 1, 8, 129, torch.float32)]
    odd = [x.cuda() for x in make(n, 2, 3, 8, 8, torch.float32)]
    half = [x.bfloat16() for x in rows]
    _, _, saved = ctx.delta_run(*half, off, save=True)
    for call in (lambda: ctx.delta_grad(saved, v), lambda: ctx.delta_grad(saved, half[2], W.bfloat16()[:1])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ctx.delta_grad(saved, half[2][:3]), lambda: ctx.delta_grad(saved, half[2], W)):
        with pytest.raises(ValueError):
            call()
    short = P.DeltaSaved(*saved.args[:-1], saved.args[-1][:-256])
    for call, status in ((lambda: ctx.delta_run(*rows, off, save=True), "UNSUPPORTED"), (lambda: ctx.delta_grad(short, half[2]), "INVALID_ARG"), (lambda: ctx.delta_run(*wide, off), "UNSUPPORTED"), (lambda: ctx.delta_run(*tall, off), "UNSUPPORTED"), (lambda: ctx.delta_step(*wide, torch.zeros(n, 1, 8, 129).cuda()), "UNSUPPORTED"), (lambda: ctx.delta_step(*tall, torch.zeros(n, 1, 129, 8).cuda()), "UNSUPPORTED"),
                         (lambda: ctx.delta_step(*odd, torch.zeros(n, 3, 8, 8).cuda()), "INVALID_ARG"), (lambda: ctx.delta_step(*rows, W[:5]), "INVALID_ARG"),
                         (lambda: ctx.delta_run(q, k, v, g, b, off, out=v), "INVALID_ARG"), (lambda: ctx.delta_run(q, k, v, g, b, off, scale=math.inf), "INVALID_ARG")):
        with pytest.raises(P.WpsgdError) as e:
            call()
        assert e.value.status_name == status
