"""Operators on whole sets of rows with so much work that every loop of their kernels goes round several times, in every form that the library
chooses from, against their formulas in 64 bits (on the GPU, by torch). Tolerances count roundings (u = 2^-24 for fp32, 2^-8 for bf16 results)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HINGE, LOGISTIC, SQUARED = 0, 1, 2
U = 2.0 ** -24
BLOCK = 128
SMS = 148


@pytest.fixture(scope="module")
def P(wpsgd_lib):
    import paper_1708_04801_b200 as pkg

    return pkg


def blocks(d):
    return -(-d // BLOCK)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(shape, seed, scale=1.0):
    return torch.randn(shape, generator=gen(seed), device="cuda") * scale


def spaced(t, ld, offset=0):
    """The same values in rows `ld` elements apart, `offset` elements into their storage; NaN between the rows."""
    n, d = t.shape
    flat = torch.full((offset + n * ld,), float("nan"), dtype=t.dtype, device="cuda")
    v = flat[offset:].view(n, ld)[:, :d]
    v.copy_(t)
    return v


# ---- 8-bit rows ------------------------------------------------------------------------------------------------------------
def pack_reference(x):
    """The definition: largest magnitude, quotient, product, rounding, one IEEE operation at a time."""
    n, d = x.shape
    x = x.float()
    a = torch.nn.functional.pad(x, (0, blocks(d) * BLOCK - d)).view(n, -1, BLOCK).abs().amax(2).clamp_min(2.0 ** -100)
    quotient = torch.div(torch.full_like(a, 448.0), a)
    return (x * quotient.repeat_interleave(BLOCK, 1)[:, :d]).to(torch.float8_e4m3fn), torch.div(a, torch.full_like(a, 448.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,ld,offset", [
    (9000, 999, 999, 0), (30000, 600, 600, 0), (50000, 384, 384, 0), (20000, 1152, 1160, 8), (40000, 321, 322, 1), (200000, 24, 24, 0), (5000, 8200, 8200, 0),
    (131072, 129, 129, 0),
])
def test_rows_packed_over_several_steps_are_the_definition_bit_for_bit(P, dtype, n, d, ld, offset):
    # a step packs 18944 blocks (bf16 rows on 16 bytes: 37888)
    x = spaced((normal((n, d), n + d) * torch.exp(normal((n, 1), 3))).to(dtype), ld, offset)
    with P.Context(1, d) as ctx:
        q, s = ctx.quantize_rows(x)
        again, _ = ctx.quantize_rows(x)
        ctx.check()
    assert n * blocks(d) > 37888
    wq, ws = pack_reference(x)
    assert torch.equal(s, ws)
    assert torch.equal(q.view(torch.uint8), wq.view(torch.uint8)) and torch.equal(q.view(torch.uint8), again.view(torch.uint8))


# ---- margins ---------------------------------------------------------------------------------------------------------------
def packed(x):
    """Packed by torch, rows that start on 16 bytes; the padding holds NaN codes."""
    n, d = x.shape
    q, s = pack_reference(x)
    buf = torch.full((n, (d + 15) // 16 * 16), 0x7f, dtype=torch.uint8, device="cuda")
    buf[:, :d] = q.view(torch.uint8)
    return buf.view(torch.float8_e4m3fn)[:, :d], s


def values(q, s):
    return q.float().double() * s.double().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def form(n, m, d):
    """(models of a tile, blocks of a cluster, tiles) by the rule of the library, so that each case below says which form it runs."""
    nb, best = blocks(d), None
    for bn, most in ((16, 8), (32, 8), (64, 4), (128, 4), (256, 1)):
        tiles = -(-n // 128) * -(-m // bn)
        for splits in (1, 2, 4, 8):
            if splits > 1 and (splits > most or tiles * splits > SMS or nb < 2 * splits):
                continue
            cycles = -(-tiles // SMS) * (-(-nb // splits) * max(2 * bn, (128 + bn) * BLOCK // 40, 600) + 12 * bn) + (5000 if splits > 1 else 0)
            if best is None or cycles < best[0]:
                best = (cycles, bn, splits, tiles)
    return best[1:]


def check_margins(z, q, s, p, t, dtype):
    # a block's 128 products are exact in fp32, its sum takes 127 additions of at most 2 u each (truncated or rounded); scale product, its
    # product with the sum and the sum over the blocks (in up to 8 parts): nb + 10 roundings
    b, nb = values(p, t), blocks(q.shape[1])
    for at in range(0, q.shape[0], 8192):
        a = values(q[at:at + 8192], s[at:at + 8192])
        want, size = a @ b.T, a.abs() @ b.abs().T
        tol = (127 * 2 + nb + 10) * U * size
        if dtype == torch.bfloat16:
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
        err = (z[at:at + 8192].double() - want).abs()
        assert bool((err <= tol + 1e-300).all()), float((err / (tol + 1e-300)).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,m,d,bn,splits,several", [
    (65000, 3, 449, 16, 1, True), (6007, 2, 3522, 16, 2, False), (4622, 15, 5000, 16, 4, False), (1, 188, 13741, 16, 8, False),
    (554, 897, 149, 32, 1, False), (46384, 18, 176, 32, 1, True), (42804, 74, 59, 32, 1, True), (4854, 17, 3899, 32, 2, False), (1998, 55, 1530, 32, 4, False),
    (50, 454, 3588, 32, 8, False),
    (320, 1726, 373, 64, 1, False), (3087, 803, 120, 64, 1, True), (52604, 134, 45, 64, 1, True), (5556, 43, 3043, 64, 2, False), (2653, 41, 3685, 64, 4, False),
    (18751, 103, 424, 128, 1, False), (5151, 840, 29, 128, 1, True), (44155, 324, 118, 128, 1, True), (8091, 1559, 5423, 128, 1, True), (296, 1893, 4588, 128, 2, False),
    (169, 1679, 2302, 128, 4, False),
    (4137, 902, 771, 256, 1, False), (9340, 837, 37, 256, 1, True), (34112, 600, 512, 256, 1, True), (28626, 1573, 1518, 256, 1, True),
])
def test_margins_in_every_form(P, dtype, n, m, d, bn, splits, several):
    got = form(n, m, d)
    assert got[:2] == (bn, splits) and (got[2] > SMS) == several
    q, s = packed(normal((n, d), 5 * n + d))
    p, t = packed(normal((m, d), 7 * m + d) * torch.exp(normal((m, 1), 2)))
    with P.Context(1, d) as ctx:
        z = ctx.margins_fp8(q, s, p, t, dtype=dtype)
        again = ctx.margins_fp8(q, s, p, t, dtype=dtype)
        ctx.check()
    check_margins(z, q, s, p, t, dtype)
    assert torch.equal(z, again)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,m,d,bn,ld,offset", [(30000, 25, 300, 32, 27, 1), (3087, 803, 120, 64, 803, 0), (18751, 103, 260, 128, 106, 3), (9340, 837, 200, 256, 838, 2)])
def test_margins_in_every_width_into_rows_of_any_stride(P, dtype, n, m, d, bn, ld, offset):
    assert form(n, m, d)[0] == bn
    q, s = packed(normal((n, d), 1))
    p, t = packed(normal((m, d), 2))
    buf = torch.full((offset + (n + 2) * ld,), 123.0, dtype=dtype, device="cuda")
    z = buf[offset:offset + n * ld].view(n, ld)[:, :m]
    with P.Context(1, d) as ctx:
        ctx.margins_fp8(q, s, p, t, out=z)
        ctx.check()
    check_margins(z, q, s, p, t, dtype)
    rest = buf.clone()
    rest[offset:offset + n * ld].view(n, ld)[:, :m] = 123.0
    assert bool((rest == 123.0).all())


# ---- objective and gradient --------------------------------------------------------------------------------------------------
def gradient_sums(x, y, w, loss):
    """Sums over the rows of x (64 bits): losses, wrong signs, gradient, and bounds of what fp32 margins and sums make of them."""
    y = y.double()
    n, d = x.shape
    z, wx = x @ w, x.abs() @ w.abs()
    if loss == HINGE:
        value, g, g1 = (1 - y * z).clamp_min(0), torch.where(y * z < 1, -y, torch.zeros_like(y)), torch.zeros_like(y)
    elif loss == LOGISTIC:
        value, g, g1 = torch.nn.functional.softplus(-y * z, threshold=1e9), -y / (1 + torch.exp(y * z)), y * y / 4
    else:
        value, g, g1 = (z - y) ** 2 / 2, z - y, torch.ones_like(y)
    dz = (d + 8) * U * wx  # a margin: a product takes part in at most d + 8 additions
    slope = torch.where(g != 0, g.abs(), y.abs() if loss == HINGE else g.abs())
    return (value.sum(), ((z >= 0) != (y >= 0)).double().sum(), x.T @ g, value.abs().sum(), (slope * dz + g1 * dz * dz).sum(),
            x.abs().T @ g.abs(), x.abs().T @ (g1 * dz))


def check_gradient(out, grad, rows, n, d, y, w, lam, loss, adds, step=16384):
    """rows(a, b): rows a to b in 64 bits. adds: additions in fp32 that a row's part of the gradient takes part in."""
    w = w.double()
    parts = [gradient_sums(rows(a, min(a + step, n)), y[a:a + step], w, loss) for a in range(0, n, step)]
    value, wrong, g, size, tol_o, gx, tol_g = (sum(p[i] for p in parts) for i in range(7))
    objective, want = lam / 2 * w @ w + value / n, lam * w + g / n
    assert abs(float(out[0]) - float(objective)) <= float(tol_o / n + 2 * U * objective.abs() + 1e-12 * size / n)
    assert float(out[1]) == float((wrong / n).float())
    # the derivative: 8 roundings, its product with a scale and an element 2; the result 2
    tol = ((adds + 10) * U * gx + tol_g) / n + 2 * U * want.abs()
    err = (grad.double() - want).abs()
    assert bool((err <= tol + 1e-300).all()), float((err / (tol + 1e-300)).max())


def problem(n, d, loss, seed=0):
    x = normal((n, d), seed + 1) / math.sqrt(d) * torch.exp(0.5 * normal((1, d), seed + 2))
    w = normal((d,), seed + 3)
    score = x @ w + 0.5 * normal((n,), seed + 4)
    y = score if loss == SQUARED else torch.where(score >= 0, 1.0, -1.0)
    return x, y, 0.8 * w + 0.2 * normal((d,), seed + 5)


V = {"f32": 4, "bf16": 8, "e4m3": 16}   # elements of a 16-byte unit
WIDTHS = [4, 8, 16, 32, 64, 128, 256, 512, 1024, 2048]  # units of a row: each up to here has a form of its own


def rounds(kind, feed, units, n):
    """How often a group of the one-pass kernel takes rows, by the library's choice of threads per row and rows at a time."""
    r = 4 if V[kind] == 16 or (V[kind] == 8 and feed == "elements") else 8
    g, r = {4: (4, 4), 512: (256, r // 2), 1024: (512, r // 2), 2048: (512, 2)}.get(units, (units, r))
    if units == 512 and V[kind] == 8 and feed == "elements":
        g, r = 512, 2 * r
    groups, per_sm = max(g, 256) // g, 1 if g > 256 else 2
    return n / (min(296, SMS * per_sm) * groups * r)


def gradient_case(kind, feed, width):
    """(rows, columns, elements from row to row): 10 to 11 rounds, the last not full; columns that leave threads of a group without any."""
    v = V[kind]
    d = width * v - (width * v // 8 if width > 4 else v)
    d -= d % v
    d, ld = {"bulk": (d, d), "units": (d - 1, d + v), "elements": (d - 1, d + 1)}[feed]
    n = int(10.4 / rounds(kind, feed, width, 1)) + 1
    return n, d, ld


FORMS = [(k, f, u) for k in ("f32", "bf16") for f in ("bulk", "units", "elements") for u in WIDTHS] + [("e4m3", "units", u) for u in WIDTHS[:-1]]


@pytest.mark.parametrize("kind,feed,width", FORMS)
def test_gradient_in_every_form_over_many_rounds(P, kind, feed, width):
    n, d, ld = gradient_case(kind, feed, width)
    assert rounds(kind, feed, width, n) > 10   # a ring has up to 8 slots, so every slot is used again
    loss = (width.bit_length() + len(feed)) % 3
    x, y, w = problem(n, d, loss, seed=d)
    with P.Context(1, d) as ctx:
        if kind == "e4m3":
            q, s = packed(x)
            wide = spaced(s, blocks(d) + 2)
            out, grad = ctx.objective_grad_fp8(q, wide, y, w, 0.01, loss)
            again = ctx.objective_grad_fp8(q, wide, y, w, 0.01, loss)
            rows = lambda a, b: values(q[a:b], s[a:b])
        else:
            x = spaced(x.to(torch.bfloat16 if kind == "bf16" else torch.float32), ld, 1 if feed == "elements" else 0)
            out, grad = ctx.objective_grad(x, y, w, 0.01, loss)
            again = ctx.objective_grad(x, y, w, 0.01, loss)
            rows = lambda a, b: x[a:b].double()
        ctx.check()
    # 11 rounds of 8 rows in a thread, then the groups of a block (64 at most), then 64 bits
    check_gradient(out, grad, rows, n, d, y, w, 0.009999999776482582, loss, adds=11 * 8 + 64)
    assert torch.equal(out, again[0]) and torch.equal(grad, again[1])


@pytest.mark.parametrize("kind,n,d,ld", [("f32", 66000, 8193, 8193), ("f32", 131500, 8200, 8200), ("bf16", 66000, 16392, 16392), ("bf16", 65537, 17001, 17002),
                                         ("e4m3", 65836, 16400, 0), ("e4m3", 131073, 16385, 0)])
def test_gradient_of_wide_rows_over_more_than_one_step(P, kind, n, d, ld):
    # rows too wide for one pass are taken 65536 at a time, each step adding to the one before
    w, y = normal((d,), 1), torch.where(normal((n,), 2) >= 0, 1.0, -1.0)
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[kind]
    store = torch.empty(n, ld or (d + 15) // 16 * 16, dtype=dtype, device="cuda")
    scales = torch.empty(n, blocks(d), device="cuda")
    x = store[:, :d]
    for a in range(0, n, 8192):
        part = normal((min(8192, n - a), d), a + 3) / math.sqrt(d)
        if kind == "e4m3":
            q, scales[a:a + 8192] = pack_reference(part)
            x[a:a + 8192].view(torch.uint8).copy_(q.view(torch.uint8))
        else:
            x[a:a + 8192].copy_(part)
    with P.Context(1, d) as ctx:
        if kind == "e4m3":
            out, grad = ctx.objective_grad_fp8(x, scales, y, w, 0.01, LOGISTIC)
            rows = lambda a, b: values(x[a:b], scales[a:b])
        else:
            out, grad = ctx.objective_grad(x, y, w, 0.01, LOGISTIC)
            rows = lambda a, b: x[a:b].double()
        ctx.check()
    # 256 columns a block, 1184 blocks, so 65536 rows in 1184 / (d / 256) parts; as often as there are steps
    parts = 1184 // -(-d // 256)
    check_gradient(out, grad, rows, n, d, y, w, 0.009999999776482582, LOGISTIC, adds=-(-n // 65536) * (-(-65536 // parts) + 1), step=4096)


# ---- norm and clipping -------------------------------------------------------------------------------------------------------
def check_clip(norm, outs, grads, max_norm):
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    f = max_norm / want if want > max_norm else 1.0
    # squares of 32 elements at most in fp32 (2 roundings of products and sums each at most 32 u), the rest in fp64; half of it in the root
    assert abs(float(norm) - want) <= 18 * U * want
    for o, g in zip(outs, grads):
        s = g.double() * f
        tol = (20 * U + (2.0 ** -8 if o.dtype == torch.bfloat16 else 0)) * s.abs()
        assert bool(((o.double() - s).abs() <= tol).all())


CLIP_LISTS = {
    # elements of each tensor; chunks are 8192 elements, blocks 1184 at most
    "short, 9 chunks": [8192 * 8 + 5], "short, 16 chunks": [30000, 90000, 1, 700], "short, 16 tensors": [5000] * 16, "17 chunks": [8192 * 16 + 1],
    "one of several chunks per block": [40000037], "few": [11000003, 1, 9000001, 17, 20000000], "32 mixed": [1000003 + 8191 * i for i in range(32)],
    "33 mixed": [1000003 + 8191 * i for i in range(33)], "many of several chunks": [20001 + i for i in range(1100)],
    "three launches": [9000 + (i * 37) % 500 for i in range(2500)],
}


@pytest.mark.parametrize("place", ["in place", "apart"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", list(CLIP_LISTS))
def test_clip_with_several_chunks_per_block(P, place, kind, sizes):
    sizes = CLIP_LISTS[sizes]
    types = [torch.float32 if kind == "f32" or (kind == "mixed" and i % 2 == 0) else torch.bfloat16 for i in range(len(sizes))]
    kept, grads, outs = [], [], []
    pools = {t: torch.full((sum(n for n, u in zip(sizes, types) if u == t) + 2,), 9.0, dtype=t, device="cuda") for t in set(types)}
    at = {t: 1 for t in pools}
    for i, (n, t) in enumerate(zip(sizes, types)):
        kept.append((normal((n,), i) * math.exp(0.3 * (i % 7))).to(t))
        grads.append(kept[-1].clone())
        outs.append(pools[t][at[t]:at[t] + n])
        at[t] += n
    lists = P.GradList(grads) if place == "in place" else P.GradList(grads, outs)
    with P.Context(1, 8) as ctx:
        norm = ctx.grad_norm(lists)
        max_norm = 0.3 * float(norm)
        got = ctx.clip_grad_norm(lists, max_norm)
        ctx.check()
    assert torch.equal(norm, got)
    check_clip(got, lists.out, kept, max_norm)
    if place == "apart":
        assert all(torch.equal(g, k) for g, k in zip(grads, kept))
        assert all(float(p[0]) == 9.0 and float(p[-1]) == 9.0 for p in pools.values())
