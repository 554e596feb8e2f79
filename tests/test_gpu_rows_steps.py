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
