"""Operators on whole sets of rows, through the public entry points, against their formulas in 64 bits: 8-bit rows, margins of many
models, objective with gradient, norm and clipping. Tolerances count roundings (u = 2^-24 for fp32, 2^-8 for bf16 results): they
are bounds of the error, computed from the inputs beside each comparison."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HINGE, LOGISTIC, SQUARED = 0, 1, 2
U = 2.0 ** -24
BLOCK = 128


@pytest.fixture(scope="module")
def P(wpsgd_lib):
    import paper_1708_04801_b200 as pkg

    return pkg


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, seed, scale=1.0):
    return torch.randn(shape, generator=gen(seed)) * scale


def blocks(d):
    return -(-d // BLOCK)


def pack_reference(x):
    """The definition in fp32 on the host: amax, reciprocal, product and rounding as specified, one operation at a time."""
    n, d = x.shape
    p = torch.nn.functional.pad(x.float(), (0, blocks(d) * BLOCK - d)).view(n, -1, BLOCK).abs()
    a = torch.where(torch.isnan(p), torch.zeros(()), p).amax(2).clamp_min(2.0 ** -100)
    q = (x.float() * torch.div(torch.full_like(a, 448.0), a).repeat_interleave(BLOCK, 1)[:, :d]).to(torch.float8_e4m3fn)
    return q, a / 448.0


def values(q, s):
    return q.float().double() * s.double().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def strided(t, pad, offset=0):
    """The same values on the GPU in rows `pad` elements apart from each other, the first `offset` elements into its storage."""
    n, d = t.shape
    flat = torch.full((offset + n * (d + pad),), 77.0).to(t.dtype).cuda()
    v = flat[offset:].view(n, d + pad)[:, :d]
    v.copy_(t)
    return v


# ---- 8-bit rows ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,pad,offset", [
    (1, 1, 0, 0), (3, 7, 0, 0), (5, 128, 0, 0), (5, 129, 7, 1), (64, 64, 0, 0), (37, 1000, 24, 0), (33, 999, 0, 0), (2, 4096, 0, 8),
    (700, 256, 0, 3), (1, 8192, 0, 0), (9, 132, 0, 0),
])
def test_quantize_rows_is_the_definition_bit_for_bit(P, dtype, n, d, pad, offset):
    x = (normal((n, d), n * d) * torch.exp(normal((n, 1), 3))).to(dtype)
    with P.Context(1, d) as ctx:
        q, s = ctx.quantize_rows(strided(x, pad, offset))
        ctx.check()
    wq, ws = pack_reference(x)
    assert q.stride(0) % 16 == 0 and q.dtype == torch.float8_e4m3fn
    assert torch.equal(s.cpu(), ws)
    assert torch.equal(q.cpu().view(torch.uint8), wq.view(torch.uint8))


def test_quantize_rows_special_values(P):
    x = torch.zeros(6, 200)
    x[1] = 1e-40                       # subnormal: scaled as if the largest were 2^-100
    x[2, 0] = 3.4e38
    x[3, 5] = float("nan")
    x[3, 6] = 2.0
    x[4, 150] = float("inf")
    x[4, 3] = 1.0
    x[5] = torch.linspace(-448, 448, 200)
    with P.Context(1, 200) as ctx:
        q, s = ctx.quantize_rows(x.cuda())
        ctx.check()
    wq, ws = pack_reference(x)
    assert torch.equal(s.cpu(), ws)
    got, want = q.cpu().float(), wq.float()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())
    assert torch.isinf(s[4, 1]) and torch.isnan(got[4, 150]) and torch.isnan(got[3, 5]) and got[3, 6] == 448.0


def test_quantize_rows_leaves_the_padding(P):
    x = normal((40, 100), 1)
    q = torch.full((40, 128), 0x5a, dtype=torch.uint8).cuda()
    s = torch.full((40, 3), -1.0).cuda()
    with P.Context(1, 100) as ctx:
        ctx.quantize_rows(x.cuda(), q[:, :100], s[:, :1])
        ctx.check()
    wq, ws = pack_reference(x)
    assert torch.equal(q[:, :100].cpu(), wq.view(torch.uint8)) and torch.equal(s[:, :1].cpu(), ws)
    assert bool((q[:, 100:] == 0x5a).all()) and bool((s[:, 1:] == -1.0).all())


# ---- margins -----------------------------------------------------------------------------------------------------------
def packed(x, pad=0):
    """Packed on the host, on the GPU with rows `pad` bytes (a multiple of 16) further apart; the padding holds NaN codes."""
    q, s = pack_reference(x)
    n, d = x.shape
    width = (d + 15) // 16 * 16 + pad
    buf = torch.full((n, width), 0x7f, dtype=torch.uint8)
    buf[:, :d] = q.view(torch.uint8)
    return q, s, buf.cuda().view(torch.float8_e4m3fn)[:, :d], s.cuda()


def check_margins(z, q, s, p, t, dtype):
    a, b = values(q, s), values(p, t)
    want, size = a @ b.T, a.abs() @ b.abs().T
    nb = blocks(q.shape[1])
    # a block's 128 products are exact in fp32, its sum takes 127 additions of at most 2 u each (truncated or rounded); scale product,
    # its product with the sum, and the sum over the blocks: nb + 2 roundings
    tol = (127 * 2 + nb + 2) * U * size
    if dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    err = (z.double().cpu() - want).abs()
    assert bool((err <= tol + 1e-300).all()), float((err / (tol + 1e-300)).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,m,d,pad", [
    (1, 1, 1, 0), (1, 1024, 256, 0), (7, 3, 64, 16), (129, 17, 128, 0), (128, 16, 129, 32), (300, 37, 999, 0), (64, 1, 4096, 0),
    (1, 5, 8200, 0), (2, 15, 5918, 0), (130, 100, 3000, 0), (257, 30, 1500, 16), (1, 40, 20000, 0), (513, 130, 640, 64), (5, 300, 33, 0), (1000, 257, 256, 0), (40, 64, 2000, 0),
])
def test_margins(P, dtype, n, m, d, pad):
    q, s, dq, ds = packed(normal((n, d), 5 * n + d), pad)
    p, t, dp, dt = packed(normal((m, d), 7 * m + d) * torch.exp(normal((m, 1), 2)), 0)
    with P.Context(1, d) as ctx:
        z = ctx.margins_fp8(dq, ds, dp, dt, dtype=dtype)
        ctx.check()
    assert z.shape == (n, m) and z.dtype == dtype
    check_margins(z, q, s, p, t, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,m,ld,offset", [(200, 33, 33, 1), (200, 32, 40, 0), (131, 129, 133, 3), (17, 256, 256, 0)])
def test_margins_into_rows_of_any_stride(P, dtype, n, m, ld, offset):
    d = 300
    q, s, dq, ds = packed(normal((n, d), 1))
    p, t, dp, dt = packed(normal((m, d), 2))
    buf = torch.full((offset + (n + 2) * ld,), 123.0, dtype=dtype).cuda()
    z = buf[offset:offset + n * ld].view(n, ld)[:, :m]
    with P.Context(1, d) as ctx:
        ctx.margins_fp8(dq, ds, dp, dt, out=z)
        ctx.check()
    check_margins(z, q, s, p, t, dtype)
    rest = buf.clone()
    rest[offset:offset + n * ld].view(n, ld)[:, :m] = 123.0
    assert bool((rest == 123.0).all())   # beside and behind the margins nothing is written


def test_margins_of_scales_with_strides_and_uint8_codes(P):
    n, m, d = 50, 20, 500
    q, s, dq, ds = packed(normal((n, d), 1))
    p, t, dp, dt = packed(normal((m, d), 2))
    wide = torch.full((n, 9), float("nan")).cuda()
    wide[:, :4] = ds
    with P.Context(1, d) as ctx:
        z = ctx.margins_fp8(dq.view(torch.uint8), wide[:, :4], dp, dt)
        ctx.check()
    check_margins(z, q, s, p, t, torch.float32)


def test_margins_of_special_values(P):
    # a NaN stays in its row (or model); an infinity in a row makes that row NaN
    n, m, d = 140, 18, 260
    x, w = normal((n, d), 1), normal((m, d), 2)
    x[3, 7] = float("nan")
    x[130, 250] = float("inf")
    w[17, 0] = float("nan")
    with P.Context(1, d) as ctx:
        Q, S = ctx.quantize_rows(x.cuda())
        M, T = ctx.quantize_rows(w.cuda())
        z = ctx.margins_fp8(Q, S, M, T).cpu()
        ctx.check()
    bad = torch.zeros(n, m, dtype=torch.bool)
    bad[3] = bad[130] = True
    bad[:, 17] = True
    assert torch.equal(torch.isnan(z), bad)


def test_margins_without_rows_or_models(P):
    with P.Context(1, 40) as ctx:
        _, _, dq, ds = packed(normal((5, 40), 1))
        none = torch.empty(0, 48, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn)[:, :40]
        no_scales = torch.empty(0, 1).cuda()
        assert ctx.margins_fp8(none, no_scales, dq, ds).shape == (0, 5)
        assert ctx.margins_fp8(dq, ds, none, no_scales).shape == (5, 0)
        q, s = ctx.quantize_rows(torch.empty(0, 40).cuda())
        assert q.shape == (0, 40) and s.shape == (0, 1)
        ctx.check()


# ---- objective and gradient ---------------------------------------------------------------------------------------------
def gradient_reference(x, y, w, lam, loss):
    """(measures, gradient, tolerance of the objective, tolerance of the gradient) in 64 bits."""
    x, y, w = x.double(), y.double(), w.double()
    n, d = x.shape
    z = x @ w
    if loss == HINGE:
        value, g, g1 = (1 - y * z).clamp_min(0), torch.where(y * z < 1, -y, torch.zeros_like(y)), torch.zeros_like(y)
    elif loss == LOGISTIC:
        value, g, g1 = torch.nn.functional.softplus(-y * z, threshold=1e9), -y / (1 + torch.exp(y * z)), y * y / 4
    else:
        value, g, g1 = (z - y) ** 2 / 2, z - y, torch.ones_like(y)
    wrong = ((z >= 0) != (y >= 0)).double()
    measures = torch.stack([lam / 2 * w @ w + value.sum() / max(n, 1), wrong.sum() / max(n, 1)])
    grad = lam * w + x.T @ g / max(n, 1)
    # a margin: a product takes part in at most d + 8 additions; the derivative: 8 roundings and what the margin's error does to it;
    # a sum over rows: at most n + 8 additions; the result: 2 roundings
    dz = (d + 8) * U * (x.abs() @ w.abs())
    tol_g = (x.abs().T @ (g.abs() * (n + 16) * U + g1 * dz)) / max(n, 1) + 2 * U * grad.abs()
    slope = torch.where(g != 0, g.abs(), y.abs() if loss == HINGE else g.abs())
    tol_o = float((slope * dz + g1 * dz * dz).sum() / max(n, 1) + 2 * U * measures[0].abs() + 1e-12 * value.abs().sum() / max(n, 1))
    return measures, grad, tol_o, tol_g


def check_gradient(out, grad, x, y, w, lam, loss):
    measures, want, tol_o, tol_g = gradient_reference(x, y, w, lam, loss)
    assert out.dtype == torch.float32 and grad.dtype == torch.float32
    assert abs(float(out[0]) - float(measures[0])) <= tol_o
    assert float(out[1]) == float(measures[1].float())
    err = (grad.double().cpu() - want).abs()
    assert bool((err <= tol_g + 1e-300).all()), float((err / (tol_g + 1e-300)).max())


def problem(n, d, loss, seed=0):
    x = normal((n, d), seed + 1) / math.sqrt(d) * torch.exp(0.5 * normal((1, d), seed + 2))
    w = normal((d,), seed + 3)
    score = x @ w + 0.5 * normal((n,), seed + 4)
    y = score if loss == SQUARED else torch.where(score >= 0, 1.0, -1.0)
    return x, y, 0.8 * w + 0.2 * normal((d,), seed + 5)


SHAPES = [(1, 1), (1, 4096), (3, 5), (300, 8), (90, 72), (1200, 520), (600, 2056), (40, 64), (257, 100), (1000, 256), (333, 999), (64, 1024), (130, 4096), (50, 8192), (20, 16384),
          (9, 20000), (70, 132), (2000, 16), (515, 40)]


@pytest.mark.parametrize("loss", [HINGE, LOGISTIC, SQUARED])
@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("n,d", SHAPES)
def test_gradient(P, loss, kind, n, d):
    x, y, w = problem(n, d, loss)
    with P.Context(1, d) as ctx:
        if kind == "e4m3":
            q, s, dq, ds = packed(x)
            out, grad = ctx.objective_grad_fp8(dq, ds, y.cuda(), w.cuda(), 0.01, loss)
            x = values(q, s)
        else:
            x = x.to(torch.bfloat16 if kind == "bf16" else torch.float32)
            out, grad = ctx.objective_grad(x.cuda(), y.cuda(), w.cuda(), 0.01, loss)
        ctx.check()
    check_gradient(out, grad, x, y, w, float(np.float32(0.01)), loss)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("d,pad,offset", [(64, 1, 0), (256, 0, 1), (512, 8, 0), (1000, 3, 5), (2050, 6, 2), (4096, 16, 8), (33, 70, 1),
                                          (1, 0, 3), (7, 101, 0), (999, 101, 3), (5001, 77, 1), (8191, 0, 1), (130, 33, 7)])
def test_gradient_of_rows_of_any_stride_and_alignment(P, kind, d, pad, offset):
    n = 77
    x, y, w = problem(n, d, LOGISTIC)
    x = x.to(torch.bfloat16 if kind == "bf16" else torch.float32)
    w_odd = torch.zeros(d + 1).cuda()[1:]
    w_odd.copy_(w)
    grad = torch.full((d + 2,), 5.0).cuda()
    with P.Context(1, d) as ctx:
        out, _ = ctx.objective_grad(strided(x, pad, offset), y.cuda(), w_odd, 0.01, LOGISTIC, grad=grad[1:d + 1])
        ctx.check()
    check_gradient(out, grad[1:d + 1], x, y, w, float(np.float32(0.01)), LOGISTIC)
    assert float(grad[0]) == 5.0 and float(grad[-1]) == 5.0


def test_gradient_of_packed_rows_with_padding(P):
    n, d = 90, 1000
    x, y, w = problem(n, d, SQUARED)
    q, s, dq, ds = packed(x, 48)   # NaN codes between the rows
    wide = torch.full((n, 11), float("nan")).cuda()
    wide[:, :8] = ds
    with P.Context(1, d) as ctx:
        out, grad = ctx.objective_grad_fp8(dq, wide[:, :8], y.cuda(), w.cuda(), 0.0, SQUARED)
        ctx.check()
    check_gradient(out, grad, values(q, s), y, w, 0.0, SQUARED)


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 700, 4096])
def test_gradient_decides_at_the_hinge_and_the_sign_as_exact_sums_do(P, kind, d):
    # margins within a few units of fp32 rounding of 1 and of 0: each decision is that of the products summed in fp64
    n = 400
    x, _, _ = problem(n, d, HINGE, seed=50)
    if kind == "e4m3":
        q, s, dq, ds = packed(x)
        xv = values(q, s)
    else:
        xt = x.to(torch.bfloat16 if kind == "bf16" else torch.float32)
        xv = xt.double()
    w = normal((d,), 9)
    z = xv @ w.double()
    y = torch.where(torch.arange(n) % 2 == 0, (1 / z).float(), (z >= 0).float() * 2 - 1)
    yz = y.double() * z
    assert float((yz[::2] - 1).abs().max()) < 2.0 ** -22   # near the hinge by construction
    with P.Context(1, d) as ctx:
        if kind == "e4m3":
            out, grad = ctx.objective_grad_fp8(dq, ds, y.cuda(), w.cuda(), 0.01, HINGE)
        else:
            out, grad = ctx.objective_grad(xt.cuda(), y.cuda(), w.cuda(), 0.01, HINGE)
        ctx.check()
    check_gradient(out, grad, xv, y, w, float(np.float32(0.01)), HINGE)


@pytest.mark.parametrize("d", [3, 300, 20000])
def test_gradient_at_zero_and_without_rows(P, d):
    x, y, _ = problem(60, d, HINGE)
    w = torch.zeros(d)
    with P.Context(1, d) as ctx:
        out, grad = ctx.objective_grad(x.cuda(), y.cuda(), w.cuda(), 0.5, HINGE)
        check_gradient(out, grad, x, y, w, 0.5, HINGE)
        w = normal((d,), 4)
        out, grad = ctx.objective_grad(x[:0].cuda(), y[:0].cuda(), w.cuda(), 0.5, HINGE)
        ctx.check()
    assert torch.equal(grad.cpu(), 0.5 * w)
    assert float(out[0]) == pytest.approx(0.25 * float(w.double() @ w.double()), rel=2 * U) and float(out[1]) == 0.0


@pytest.mark.parametrize("loss", [HINGE, LOGISTIC, SQUARED])
def test_gradient_of_values_that_are_not_finite(P, loss):
    x, y, w = problem(50, 130, loss)
    x[7, 3] = float("nan")
    with P.Context(1, 130) as ctx:
        out, grad = ctx.objective_grad(x.cuda(), y.cuda(), w.cuda(), 0.01, loss)
        ctx.check()
    assert math.isnan(float(out[0])) and bool(torch.isnan(grad).all())   # the row's margin is none, so its derivative is none


@pytest.mark.parametrize("kind", ["f32", "bf16", "two passes"])
@pytest.mark.parametrize("loss", [HINGE, LOGISTIC, SQUARED])
def test_gradient_with_a_label_or_a_row_that_is_not_a_number(P, loss, kind):
    d = 40000 if kind == "two passes" else 200
    x, y, w = problem(30, d, loss)
    x = x.to(torch.bfloat16) if kind == "bf16" else x
    for at in ("label", "row"):
        xb, yb = x.clone(), y.clone()
        if at == "label":
            yb[11] = float("nan")
        else:
            xb[29, d - 1] = float("nan")
        with P.Context(1, d) as ctx:
            out, grad = ctx.objective_grad(xb.cuda(), yb.cuda(), w.cuda(), 0.01, loss)
            ctx.check()
        assert math.isnan(float(out[0])) and bool(torch.isnan(grad).all())


@pytest.mark.parametrize("loss", [LOGISTIC, SQUARED])
def test_gradient_agrees_with_differences_of_the_objective(P, loss):
    # (c(w + h v) - c(w - h v)) / 2h = grad . v + h^2 / 6 c'''; objectives in 64 bits by the formula, the gradient by the kernel
    n, d, h = 200, 96, 1e-4
    x, y, w = problem(n, d, loss)
    v = normal((d,), 8)
    with P.Context(1, d) as ctx:
        _, grad = ctx.objective_grad(x.cuda(), y.cuda(), w.cuda(), 0.25, loss)
        ctx.check()
    def c(at):
        z = x.double() @ at
        val = torch.nn.functional.softplus(-y.double() * z, threshold=1e9) if loss == LOGISTIC else (z - y.double()) ** 2 / 2
        return 0.125 * at @ at + val.mean()
    diff = (c(w.double() + h * v.double()) - c(w.double() - h * v.double())) / (2 * h)
    _, _, _, tol_g = gradient_reference(x, y, w, 0.25, loss)
    xv = (x.double() @ v.double()).abs()
    third = float((xv ** 3).mean()) * 0.1 if loss == LOGISTIC else 0.0   # |third derivative of the logistic loss| < 0.1
    tol = float((tol_g * v.double().abs()).sum()) + h * h / 6 * third + 1e-15 / h * (1 + float(c(w.double())))
    assert abs(float(grad.double().cpu() @ v.double()) - float(diff)) <= tol


def test_gradient_of_many_rows(P):
    # more rows than one step of the two-pass kernels takes, and enough for every block of the one-pass kernel
    n, d = 70000, 24
    x, y, w = problem(n, d, LOGISTIC)
    with P.Context(1, d) as ctx:
        out, grad = ctx.objective_grad(x.cuda(), y.cuda(), w.cuda(), 0.01, LOGISTIC)
        again = ctx.objective_grad(x.cuda(), y.cuda(), w.cuda(), 0.01, LOGISTIC)
        ctx.check()
    check_gradient(out, grad, x, y, w, float(np.float32(0.01)), LOGISTIC)
    assert torch.equal(out, again[0]) and torch.equal(grad, again[1])


# ---- norm and clipping ---------------------------------------------------------------------------------------------------
def clip_reference(grads, max_norm):
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    f = max_norm / norm if norm > max_norm else 1.0
    return norm, [g.double() * f for g in grads], f


def check_clip(norm, outs, grads, max_norm):
    want, scaled, f = clip_reference([g.cpu() for g in grads], max_norm)
    # squares of 32 elements at most in fp32 (2 roundings of products and sums each at most 32 u), the rest in fp64; half of it in the root
    assert abs(float(norm) - want) <= 18 * U * want
    for o, g, s in zip(outs, grads, scaled):
        tol = (0 if f == 1.0 else 20 * U + (2.0 ** -8 if o.dtype == torch.bfloat16 else 0)) * s.abs()
        assert bool(((o.double().cpu() - s).abs() <= tol).all())


LISTS = {
    "one element": [1], "one": [1000], "empty ones": [0, 5, 0, 0, 7, 0], "ragged": [1, 2, 3, 4, 5, 8191, 8192, 8193, 100003, 17],
    "many": [1 + (i * 37) % 300 for i in range(2100)], "many equal": [64] * 33, "large": [3000001, 70000],
}


@pytest.mark.parametrize("place", ["in place", "apart", "apart, other alignment"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", list(LISTS))
def test_clip(P, place, kind, sizes):
    sizes = LISTS[sizes]
    types = [torch.float32 if kind == "f32" or (kind == "mixed" and i % 2 == 0) else torch.bfloat16 for i in range(len(sizes))]
    pools = {t: torch.empty(sum(sizes) + 8, dtype=t).cuda() for t in set(types)}
    at = {t: 1 for t in pools}
    grads, kept = [], []
    for i, (n, t) in enumerate(zip(sizes, types)):   # packed one behind the other: any alignment of elements
        v = pools[t][at[t]:at[t] + n]
        v.copy_((normal((n,), i) * math.exp(0.3 * (i % 7))).to(t))
        at[t] += n
        grads.append(v)
        kept.append(v.clone())
    outs = None
    if place != "in place":
        off = 1 if place == "apart" else 4
        opools = {t: torch.full_like(p, 9.0) for t, p in pools.items()}
        outs, at = [], {t: off for t in pools}
        for n, t in zip(sizes, types):
            outs.append(opools[t][at[t]:at[t] + n])
            at[t] += n
    lists = P.GradList(grads, outs)
    with P.Context(1, 8) as ctx:
        norm = ctx.grad_norm(lists)
        max_norm = 0.3 * float(norm)
        got = ctx.clip_grad_norm(lists, max_norm)
        ctx.check()
    assert torch.equal(norm, got)
    check_clip(got, lists.out, kept, max_norm)
    if outs is not None:
        assert all(torch.equal(g, k) for g, k in zip(grads, kept))
        for t, p in opools.items():
            assert bool((p[:off] == 9.0).all()) and bool((p[at[t]:] == 9.0).all())


@pytest.mark.parametrize("place", ["in place", "apart"])
@pytest.mark.parametrize("max_norm", ["above", "infinite", "zero"])
def test_clip_at_the_ends(P, place, max_norm):
    grads = [normal((n,), n).cuda() for n in (100, 9000)]
    kept = [g.clone() for g in grads]
    outs = None if place == "in place" else [torch.empty_like(g) for g in grads]
    limit = {"above": 1e6, "infinite": math.inf, "zero": 0.0}[max_norm]
    lists = P.GradList(grads, outs)
    with P.Context(1, 8) as ctx:
        ctx.clip_grad_norm(lists, limit)
        ctx.check()
    for o, k in zip(lists.out, kept):
        assert torch.equal(o, k if limit > 0 else torch.zeros_like(k))


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e30])
def test_norm_of_values_whose_squares_leave_fp32(P, scale):
    grads = [normal((5000,), 1, scale).cuda(), torch.zeros(40000).cuda(), normal((33,), 2, scale).cuda()]
    kept = [g.clone() for g in grads]
    with P.Context(1, 8) as ctx:
        norm = ctx.clip_grad_norm(grads, 0.5 * scale)
        ctx.check()
    check_clip(norm, grads, kept, 0.5 * scale)


def test_clip_of_values_that_are_not_finite(P):
    with P.Context(1, 8) as ctx:
        g = [torch.ones(50).cuda(), torch.ones(20000).cuda()]
        g[1][777] = float("inf")
        norm = ctx.clip_grad_norm(g, 1.0)
        assert float(norm) == math.inf
        assert bool((g[0] == 0).all()) and int(torch.isnan(g[1]).sum()) == 1
        g = [torch.ones(50).cuda(), torch.ones(20000).cuda()]
        g[1][777] = float("nan")
        kept = [t.clone() for t in g]
        assert math.isnan(float(ctx.clip_grad_norm(g, 1.0)))
        assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(g, kept))
        assert float(ctx.clip_grad_norm([], 1.0)) == 0.0 and float(ctx.grad_norm([torch.empty(0).cuda()])) == 0.0
        ctx.check()


# ---- refusals ------------------------------------------------------------------------------------------------------------
def test_refusals_of_the_c_entry_points(P, wpsgd_lib):
    lib, d, n = wpsgd_lib, 100, 4
    x = torch.zeros(n, d).cuda()
    q = torch.zeros(n, 112, dtype=torch.uint8).cuda()
    s = torch.zeros(n, 1).cuda()
    y, w, g, out = torch.ones(n).cuda(), torch.zeros(d).cuda(), torch.zeros(d).cuda(), torch.zeros(2).cuda()
    z = torch.zeros(n, n).cuda()
    with P.Context(1, d) as ctx:
        h = ctx._h
        def refused(status, fn, *args):
            args = [a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args]
            assert fn(h, *args) == status and lib.wpsgd_last_error(h)
        quant = lib.wpsgd_quantize_rows
        refused(1, quant, x, 7, d, n, q, 112, s, 1)            # element type
        refused(1, quant, x, 0, d - 1, n, q, 112, s, 1)        # stride below d
        refused(1, quant, None, 0, d, n, q, 112, s, 1)
        refused(1, quant, x, 0, d, -1, q, 112, s, 1)
        refused(1, quant, x, 0, d, n, q, 104, s, 1)            # stride not a multiple of 16
        refused(1, quant, x, 0, d, n, q, 96, s, 1)
        refused(1, quant, x, 0, d, n, q.data_ptr() + 4, 112, s, 1)
        refused(1, quant, x, 0, d, n, q, 112, s, 0)
        refused(1, quant, x, 0, d, n, q, 112, None, 1)
        refused(1, quant, x.data_ptr() + 2, 0, d, n, q, 112, s, 1)
        marg = lib.wpsgd_margins_fp8
        refused(1, marg, q, 112, s, 1, n, q, 112, s, 1, n, None, 0, n)
        refused(1, marg, q, 112, s, 1, n, q, 112, s, 1, n, z, 0, n - 1)
        refused(1, marg, q, 112, s, 1, n, q, 112, s, 1, n, z, 2, n)
        refused(1, marg, q, 112, s, 1, n, q, 104, s, 1, n, z, 0, n)
        refused(1, marg, q, 112, s, 0, n, q, 112, s, 1, n, z, 0, n)
        refused(1, marg, q, 112, s, 1, n, None, 112, s, 1, n, z, 0, n)
        refused(1, marg, q, 112, s, 1, n, q, 112, s, 1, n, z.data_ptr() + 2, 0, n)
        refused(5, marg, q, 112, s, 1, 1 << 31, q, 112, s, 1, n, z, 0, n)
        grad = lib.wpsgd_objective_grad
        refused(1, grad, x, 0, d, y, n, w, 0.1, 3, g, out)     # loss
        refused(1, grad, x, 5, d, y, n, w, 0.1, 0, g, out)
        refused(1, grad, x, 0, d, None, n, w, 0.1, 0, g, out)
        refused(1, grad, x, 0, d, y, n, w, math.nan, 0, g, out)
        refused(1, grad, x, 0, d, y, n, w, 0.1, 0, w, out)     # the gradient over the model
        refused(1, grad, x, 0, d, y, n, w, 0.1, 0, g, g)
        refused(1, grad, x, 0, d - 1, y, n, w, 0.1, 0, g, out)
        refused(1, lib.wpsgd_objective_grad_fp8, q, 100, s, 1, y, n, w, 0.1, 0, g, out)
        refused(1, lib.wpsgd_objective_grad_fp8, q, 112, s, 1, y, n, None, 0.1, 0, g, out)
        lists = P.GradList([x])
        refused(1, lib.wpsgd_clip_grad_norm, lists._h, -1.0, out)
        refused(1, lib.wpsgd_clip_grad_norm, lists._h, math.nan, out)
        refused(1, lib.wpsgd_clip_grad_norm, lists._h, 1.0, None)
        refused(1, lib.wpsgd_clip_grad_norm, lists._h, 1.0, x)         # the norm into a gradient
        refused(1, lib.wpsgd_grad_norm, lists._h, x.data_ptr() + 4 * n * d - 4)
        refused(1, lib.wpsgd_grad_norm, None, out)
        ctx.check()


def test_refusals_of_the_binding(P):
    with P.Context(1, 100) as ctx:
        x = torch.zeros(4, 100).cuda()
        q, s = ctx.quantize_rows(x)
        with pytest.raises(ValueError):
            ctx.quantize_rows(torch.zeros(4, 99).cuda())
        with pytest.raises(ValueError):
            ctx.quantize_rows(torch.zeros(100, 4).cuda().t())
        with pytest.raises(TypeError):
            ctx.quantize_rows(x.half())
        with pytest.raises(TypeError):
            ctx.quantize_rows(torch.zeros(4, 100))
        with pytest.raises(ValueError):
            ctx.margins_fp8(q, s[:3], q, s)
        with pytest.raises(ValueError):
            ctx.margins_fp8(q, s, q, s, out=torch.zeros(3, 4).cuda())
        with pytest.raises(P.WpsgdError):
            ctx.margins_fp8(torch.zeros(4, 100, dtype=torch.uint8).cuda(), s, q, s)   # rows that do not start on 16 bytes
        with pytest.raises(ValueError):
            ctx.objective_grad(x, torch.zeros(3).cuda(), torch.zeros(100).cuda(), 0.1, HINGE)
        with pytest.raises(TypeError):
            ctx.clip_grad_norm([torch.zeros(4, 4).cuda().t()], 1.0)
        with pytest.raises(P.WpsgdError):
            ctx.clip_grad_norm([x, x], 1.0)   # the same tensor twice, in place
        ctx.check()


# ---- bounded waits ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,m,d", [(300, 40, 700), (2, 15, 5918), (40000, 16, 256)])
def test_margins_report_a_wait_that_runs_out_and_the_context_stays_usable(P, n, m, d):
    q, s, dq, ds = packed(normal((n, d), 1))
    p, t, dp, dt = packed(normal((m, d), 2))
    with P.Context(1, d) as ctx:
        ctx.set_option("spin_limit", 2000)
        ctx.set_option("test_drop_block", 0)   # the first block of columns of every tile is never requested
        ctx.margins_fp8(dq, ds, dp, dt)
        with pytest.raises(P.WpsgdError) as e:
            ctx.check()
        assert e.value.status_name == "TIMEOUT"
        ctx.set_option("test_drop_block", -1)
        ctx.set_option("spin_limit", 1 << 20)
        z = ctx.margins_fp8(dq, ds, dp, dt)
        ctx.check()
    check_margins(z, q, s, p, t, torch.float32)


@pytest.mark.parametrize("n,d", [(50000, 64), (9000, 1024), (3000, 8192)])
def test_gradient_reports_a_wait_that_runs_out_and_the_context_stays_usable(P, n, d):
    x, y, w = problem(n, d, LOGISTIC)
    x, y, w = x.cuda(), y.cuda(), w.cuda()
    with P.Context(1, d) as ctx:
        want = ctx.objective_grad(x, y, w, 0.01, LOGISTIC)
        ctx.check()
        ctx.set_option("spin_limit", 2000)
        ctx.set_option("test_drop_block", 0)   # the first rows of every ring are never requested
        ctx.objective_grad(x, y, w, 0.01, LOGISTIC)
        with pytest.raises(P.WpsgdError) as e:
            ctx.check()
        assert e.value.status_name == "TIMEOUT"
        ctx.set_option("test_drop_block", -1)
        ctx.set_option("spin_limit", 1 << 20)
        again = ctx.objective_grad(x, y, w, 0.01, LOGISTIC)
        ctx.check()
    assert torch.equal(want[0], again[0]) and torch.equal(want[1], again[1])


def test_calls_on_a_destroyed_context_are_refused(P):
    x = torch.zeros(4, 100).cuda()
    ctx = P.Context(1, 100)
    q, s = ctx.quantize_rows(x)
    ctx.destroy()
    for call in (lambda: ctx.quantize_rows(x), lambda: ctx.margins_fp8(q, s, q, s), lambda: ctx.grad_norm([x]), lambda: ctx.clip_grad_norm([x], 1.0),
                 lambda: ctx.objective_grad(x, x[:, 0].contiguous(), x[0], 0.1, HINGE), lambda: ctx.objective_grad_fp8(q, s, x[:, 0].contiguous(), x[0], 0.1, HINGE)):
        with pytest.raises(P.WpsgdError) as e:
            call()
        assert e.value.status_name == "INVALID_ARG"


def test_two_graphs_of_two_contexts_replayed_at_once(P):
    # each context has its own workspace, so its graph may run beside the other's
    d, n = 700, 30000
    sides = []
    for i in range(2):
        x, y, w = (t.cuda() for t in problem(n, d, LOGISTIC, seed=10 * i))
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            ctx = P.Context(1, d, stream=stream)
            want = ctx.objective_grad(x, y, w, 0.01, LOGISTIC)
            grads = [torch.randn(200000, device="cuda") for _ in range(3)]
            outs, norm = [torch.empty_like(g) for g in grads], torch.empty(1).cuda()
            lists = P.GradList(grads, outs)
            ctx.grad_norm(lists)
            grad, out = torch.empty(d).cuda(), torch.empty(2).cuda()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                ctx.objective_grad(x, y, w, 0.01, LOGISTIC, grad=grad, out=out)
                ctx.clip_grad_norm(lists, 1.0, norm=norm)
        sides.append((stream, ctx, graph, want, grad, out, grads, outs, norm, (x, y, w, lists)))
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, _, graph, *_ in sides:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, ctx, graph, want, grad, out, grads, outs, norm, _ in sides:
        ctx.check()
        assert torch.equal(want[0], out) and torch.equal(want[1], grad)
        check_clip(norm, outs, grads, 1.0)
        del graph
        ctx.destroy()


# ---- streams, graphs, a run of them together -------------------------------------------------------------------------------
def test_first_call_inside_a_capture_is_refused_and_later_ones_are_captured(P):
    d, n = 200, 300
    x, y, w = problem(n, d, LOGISTIC)
    x, y, w = x.cuda(), y.cuda(), w.cuda()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = P.Context(1, d, stream=stream)
        grad, out, norm = torch.empty(d).cuda(), torch.empty(2).cuda(), torch.empty(1).cuda()
        clipped = torch.empty(d).cuda()
        lists = P.GradList([grad], [clipped])
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(P.WpsgdError) as e:
                ctx.objective_grad(x, y, w, 0.01, LOGISTIC, grad=grad, out=out)
            assert e.value.status_name == "STATE"
        want = ctx.objective_grad(x, y, w, 0.01, LOGISTIC)
        Q, S = ctx.quantize_rows(x)
        Z = ctx.margins_fp8(Q, S, Q, S)
        wq = ctx.objective_grad_fp8(Q, S, y, w, 0.01, LOGISTIC)[1].clone()
        graph = torch.cuda.CUDAGraph()
        Q2, S2, Z2, g2 = torch.zeros_like(Q.view(torch.uint8)), torch.zeros_like(S), torch.zeros_like(Z), torch.zeros_like(grad)
        Q2 = torch.zeros(n, 208, dtype=torch.uint8).cuda()[:, :d]
        with torch.cuda.graph(graph, stream=stream):
            ctx.quantize_rows(x, Q2, S2)
            ctx.margins_fp8(Q2, S2, Q2, S2, out=Z2)
            ctx.objective_grad_fp8(Q2, S2, y, w, 0.01, LOGISTIC, grad=g2, out=out)
            ctx.objective_grad(x, y, w, 0.01, LOGISTIC, grad=grad, out=out)
            ctx.clip_grad_norm(lists, 1e-3, norm=norm)
        for _ in range(3):
            for t in (Z2, g2, grad, clipped):
                t.fill_(-7.0)
            graph.replay()
        ctx.check()
        assert torch.equal(Z, Z2) and torch.equal(wq, g2) and torch.equal(want[1], grad) and torch.equal(want[0], out)
        check_clip(norm, [clipped], [want[1]], 1e-3)
        del graph
        ctx.destroy()


def test_context_on_a_stream_of_its_own(P):
    d, n = 256, 400
    x, y, w = problem(n, d, SQUARED)
    stream = torch.cuda.Stream()
    xd, yd, wd = x.cuda(), y.cuda(), w.cuda()
    torch.cuda.synchronize()
    with P.Context(1, d, stream=stream) as ctx:
        out, grad = ctx.objective_grad(xd, yd, wd, 0.01, SQUARED)   # current stream: the default one
        q, s = ctx.quantize_rows(xd)
        z = ctx.margins_fp8(q, s, q[:5], s[:5])
        ctx.check()                                                # waits for the context's stream
    check_gradient(out, grad, x, y, w, float(np.float32(0.01)), SQUARED)
    hq, hs = pack_reference(x)
    check_margins(z, hq, hs, hq[:5], hs[:5], torch.float32)


def test_contexts_on_two_streams_at_once(P):
    d, n = 512, 20000
    sides = []
    for i in range(2):
        x, y, w = problem(n, d, LOGISTIC, seed=100 * i)
        stream = torch.cuda.Stream()
        sides.append((x, y, w, x.cuda(), y.cuda(), w.cuda(), stream, P.Context(1, d, stream=stream)))
    torch.cuda.synchronize()
    got = [[] for _ in sides]
    for _ in range(4):
        for i, (_, _, _, xd, yd, wd, _, ctx) in enumerate(sides):
            out, grad = ctx.objective_grad(xd, yd, wd, 0.01, LOGISTIC)
            got[i].append((out, grad, ctx.grad_norm([grad])))
    for i, (x, y, w, *_, ctx) in enumerate(sides):
        ctx.check()
        for out, grad, norm in got[i]:
            check_gradient(out, grad, x, y, w, float(np.float32(0.01)), LOGISTIC)
            assert float(norm) == pytest.approx(float(grad.double().norm()), rel=18 * U)
        ctx.destroy()


def test_evaluation_and_polishing_after_the_chains(P):
    """As a program uses them together: chains on fp32 rows, the test rows packed once, the margins of every node's model and of the
    combined one in one product, then some full-gradient steps on the combined model with their gradient clipped."""
    import wpsgd_inputs as wi

    wl = wi.small(2).to("cuda")
    with P.Context(wl.k, wl.d) as ctx:
        ctx.run_workload(wl)
        v = ctx.combine()
        models = torch.cat([ctx.get_models(), v[None]])
        Q, S = ctx.quantize_rows(wl.X)
        M, T = ctx.quantize_rows(models)
        z = ctx.margins_fp8(Q, S, M, T)
        a, b = values(Q.cpu(), S.cpu()), values(M.cpu(), T.cpu())
        check_margins(z, Q.cpu(), S.cpu(), M.cpu(), T.cpu(), torch.float32)
        # each packed value is off by 2^-4 of itself or by the half step 2^-10 of the subnormal codes, times the scale (and 2 u)
        exact = wl.X.cpu().double() @ models.cpu().double().T
        def off(full, part, scales):
            return (full.double().cpu().abs() * (2.0 ** -4 + 4 * U) + 2.0 ** -10 * scales.cpu().double().repeat_interleave(BLOCK, 1)[:, :wl.d])
        dx, dw = off(wl.X, a, S), off(models, b, T)
        bound = dx @ models.cpu().double().abs().T + wl.X.cpu().double().abs() @ dw.T + dx @ dw.T
        assert bool(((a @ b.T - exact).abs() <= bound).all())
        out0, _ = ctx.objective_grad(wl.X, wl.y, v, wl.lam, wl.loss)
        both = ctx.objective(wl.X, wl.y, v, wl.lam, wl.loss)
        assert float(out0[0]) == pytest.approx(float(both[0]), rel=(wl.d + 8) * U) 
        for _ in range(3):
            out, grad = ctx.objective_grad(wl.X, wl.y, v, wl.lam, wl.loss)
            check_gradient(out, grad, wl.X.cpu(), wl.y.cpu(), v.cpu(), float(np.float32(wl.lam)), wl.loss)
            kept = grad.clone()
            norm = ctx.clip_grad_norm([grad], 0.01)
            check_clip(norm, [grad], [kept], 0.01)
            v = v - grad
        ctx.set_models(v)
        assert torch.equal(ctx.get_models(), v.expand(wl.k, wl.d))
        ctx.check()
