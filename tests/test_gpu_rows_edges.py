"""Operators on whole sets of rows where their calls could go wrong: lists that leave blocks empty, limits of waits, extreme magnitudes,
overlapping and unaligned arguments. Against the formulas in 64 bits; tolerances count roundings (u = 2^-24)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def P(wpsgd_lib):
    import paper_1708_04801_b200 as pkg

    return pkg


# ---- short lists: one cluster of blocks ------------------------------------------------------------------------------------
@pytest.mark.parametrize("tensors", [1, 2, 7, 16])
def test_norms_of_short_lists_call_after_call(P, tensors):
    # with fewer chunks than blocks, the blocks without any reach the exchange of sums at once: every call finds all sums
    g = torch.Generator().manual_seed(tensors)
    grads = [torch.randn(500 + 3 * i, generator=g).cuda() for i in range(tensors)]
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    with P.Context(1, 8) as ctx:
        lists = P.GradList(grads)
        norms = torch.cat([ctx.grad_norm(lists) for _ in range(2000)])
        ctx.check()
    # squares of at most 16 elements a thread in fp32 (products and additions: 16 u), half of it in the root, rounded once; the rest in fp64
    assert bool((norms == norms[0]).all()) and abs(float(norms[0]) - want) <= 10 * U * want


# ---- waits that run out ------------------------------------------------------------------------------------------------------
def rows_problem(n, d, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, d, generator=g, device="cuda") / math.sqrt(d)
    w = torch.randn(d, generator=g, device="cuda")
    return x, torch.where(torch.randn(n, generator=g, device="cuda") >= 0, 1.0, -1.0), w


@pytest.mark.parametrize("round_lost", [1, 3, 6])
@pytest.mark.parametrize("n,d", [(600000, 16), (300000, 64), (40000, 1024), (9000, 4096), (4000, 8192)])
def test_gradient_after_a_wait_that_runs_out_in_the_middle(P, n, d, round_lost):
    # the rows of a later round never come: by then every slot of the rings has been used and others are on their way
    x, y, w = rows_problem(n, d)
    with P.Context(1, d) as ctx:
        want = ctx.objective_grad(x, y, w, 0.01, 1)
        ctx.check()
        ctx.set_option("spin_limit", 2000)
        ctx.set_option("test_drop_block", round_lost)
        ctx.objective_grad(x, y, w, 0.01, 1)
        with pytest.raises(P.WpsgdError) as e:
            ctx.check()
        assert e.value.status_name == "TIMEOUT"
        ctx.set_option("test_drop_block", -1)
        ctx.set_option("spin_limit", 1 << 20)
        again = ctx.objective_grad(x, y, w, 0.01, 1)
        ctx.check()
    assert torch.equal(want[0], again[0]) and torch.equal(want[1], again[1])


def packed_normal(n, d, seed):
    """8-bit rows and scales made by torch on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, d, generator=g, device="cuda")
    nb = -(-d // 128)
    a = torch.nn.functional.pad(x, (0, nb * 128 - d)).view(n, nb, 128).abs().amax(2)
    q = torch.zeros(n, -(-d // 16) * 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :d]
    q.copy_((x * (448.0 / a).repeat_interleave(128, 1)[:, :d]).to(torch.float8_e4m3fn))
    return q, a / 448.0


LIMITS = [1, 2, 3, 5, 8, 13, 21, 34, 55, 89, 144, 1000]


@pytest.mark.parametrize("n,d", [(600000, 16), (40000, 1024), (9000, 4096), (4000, 8192)])
def test_gradient_with_waits_that_run_out_here_and_there(P, n, d):
    # limits so low that rows on their way are given up: reported, or the result is whole; what comes after is as before
    x, y, w = rows_problem(n, d)
    with P.Context(1, d) as ctx:
        want = ctx.objective_grad(x, y, w, 0.01, 1)
        ctx.check()
        for limit in LIMITS:
            ctx.set_option("spin_limit", limit)
            got = ctx.objective_grad(x, y, w, 0.01, 1)
            try:
                ctx.check()
                assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
            except P.WpsgdError as e:
                assert e.status_name == "TIMEOUT"
            ctx.set_option("spin_limit", 1 << 20)
            again = ctx.objective_grad(x, y, w, 0.01, 1)
            ctx.check()
            assert torch.equal(want[0], again[0]) and torch.equal(want[1], again[1])


@pytest.mark.parametrize("n,m,d", [(2, 15, 5918), (40000, 16, 1024), (9000, 1000, 2000)])
def test_margins_with_waits_that_run_out_here_and_there(P, n, m, d):
    q, s = packed_normal(n, d, 1)
    p, t = packed_normal(m, d, 2)
    with P.Context(1, d) as ctx:
        want = ctx.margins_fp8(q, s, p, t)
        ctx.check()
        for limit in LIMITS:
            ctx.set_option("spin_limit", limit)
            got = ctx.margins_fp8(q, s, p, t)
            try:
                ctx.check()
                assert torch.equal(want, got)
            except P.WpsgdError as e:
                assert e.status_name == "TIMEOUT"
            ctx.set_option("spin_limit", 1 << 20)
            again = ctx.margins_fp8(q, s, p, t)
            ctx.check()
            assert torch.equal(want, again)


# ---- decisions at the jumps, at the ends of fp32's range ----------------------------------------------------------------------
HINGE = 0
KINDS = ["f32", "bf16", "e4m3", "two passes"]


def rows_of(kind, x):
    """(rows and scales as the entry points take them, their values in 64 bits)"""
    if kind == "e4m3":
        n, d = x.shape
        nb = -(-d // 128)
        a = torch.nn.functional.pad(x, (0, nb * 128 - d)).view(n, nb, 128).abs().amax(2)
        q = torch.zeros(n, -(-d // 16) * 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :d]
        q.copy_((x * torch.div(torch.full_like(a, 448.0), a).repeat_interleave(128, 1)[:, :d]).to(torch.float8_e4m3fn))
        s = a / 448.0
        return (q, s), q.float().double() * s.double().repeat_interleave(128, 1)[:, :d]
    x = x.to(torch.bfloat16 if kind == "bf16" else torch.float32)
    return (x,), x.double()


def decided(ctx, kind, rows, values, y, w):
    """Error count and gradient (lambda 0) are those of margins summed in 64 bits."""
    fn = ctx.objective_grad_fp8 if kind == "e4m3" else ctx.objective_grad
    out, grad = fn(*rows, y, w, 0.0, HINGE)
    ctx.check()
    n, yd = values.shape[0], y.double()
    z = values @ w.double()
    wrong = ((z >= 0) != (yd >= 0)).double().mean()
    assert float(out[1]) == float(wrong.float())
    g = torch.where(yd * z < 1, -yd, torch.zeros_like(yd))
    want, size = values.T @ g / n, values.abs().T @ g.abs() / n
    # a row's part of the gradient: its product and at most n additions; the result 2. Divided by the largest: squares of 2^-80 are out of range
    assert bool(((grad.double() - want).abs() <= (n + 4) * U * size).all())


def width(kind, d):
    return 8200 + d if kind == "two passes" else d


@pytest.mark.parametrize("power", [0, -60, -80, -90, 60])
@pytest.mark.parametrize("d", [64, 700])
@pytest.mark.parametrize("kind", KINDS)
def test_hinge_is_decided_as_exact_sums_do_whatever_the_size_of_the_rows(P, kind, d, power):
    # rows of size 2^power on a model of size 2^-power, margins within a few units of rounding of the hinge
    n, d = 400, width(kind, d)
    g = torch.Generator(device="cuda").manual_seed(d + power)
    rows, values = rows_of(kind, torch.randn(n, d, generator=g, device="cuda") / math.sqrt(d) * 2.0 ** power)
    w = torch.randn(d, generator=g, device="cuda") * 2.0 ** -power
    y = (1 / (values @ w.double())).float()
    assert float((y.double() * (values @ w.double()) - 1).abs().max()) < 2.0 ** -22
    with P.Context(1, d) as ctx:
        decided(ctx, kind, rows, values, y, w)


@pytest.mark.parametrize("power", [0, -60, -80, -90, 60])
@pytest.mark.parametrize("d", [64, 700])
@pytest.mark.parametrize("kind", KINDS)
def test_signs_are_those_of_exact_sums_whatever_the_size_of_the_rows(P, kind, d, power):
    # the second half of each row undoes the first but for a rounding: what is left of the margin is smaller than the error of an fp32 sum
    n, d = 400, width(kind, d) // 2 * 2
    g = torch.Generator(device="cuda").manual_seed(d + power)
    half = torch.randn(n, d // 2, generator=g, device="cuda")
    w = torch.randn(d, generator=g, device="cuda")
    w[d // 2:] = w[:d // 2] * (1 + torch.randn(d // 2, generator=g, device="cuda") * 2.0 ** -23)
    rows, values = rows_of(kind, torch.cat([half, -half], 1) * 2.0 ** power)
    if kind == "e4m3":   # scales of blocks that hold different columns differ: only one block per half is undone
        rows[1][:] = rows[1][:, :1]
        values = rows[0].float().double() * rows[1].double().repeat_interleave(128, 1)[:, :d]
    y = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, -1.0)
    with P.Context(1, d) as ctx:
        decided(ctx, kind, rows, values, y, w)


@pytest.mark.parametrize("loss", [0, 1, 2])
@pytest.mark.parametrize("kind", KINDS)
def test_margins_whose_partial_sums_leave_fp32(P, kind, loss):
    # products of 2e38 and -1.9e38 in turn: sums of every other one leave fp32, the margin does not
    n, d = 20, 40
    w = torch.where(torch.arange(d) % 2 == 0, 1.0e19, -0.95e19).cuda()
    x = torch.full((n, d), 2.0e19).cuda()
    if kind == "two passes":
        x, w = (torch.nn.functional.pad(t, (0, 8200 - d)) for t in (x, w))
        d = 8200
    rows, values = rows_of(kind, x)
    y = torch.ones(n, device="cuda")
    z = values @ w.double()
    assert bool((z > 1e38).all()) and bool((z < 3e38).all())
    with P.Context(1, d) as ctx:
        fn = ctx.objective_grad_fp8 if kind == "e4m3" else ctx.objective_grad
        out, grad = fn(*rows, y, w, 0.0, loss)
        ctx.check()
    assert float(out[1]) == 0.0
    if loss == 2:   # (z - y) x leaves fp32, and the square of z - y
        assert math.isinf(float(out[0])) and bool(torch.isinf(grad[:40]).all())
    else:
        assert float(out[0]) == 0.0 and bool((grad == 0).all())


# ---- clipping --------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("place", ["in place", "apart"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e-7, 1e-20])
@pytest.mark.parametrize("sizes", [[7], [5000, 3, 9001], [700000, 20001], [1500] * 40])
def test_clip_by_a_factor_below_the_normal_numbers_of_fp32(P, sizes, max_norm, dtype, place):
    # gradients up to 3e38 brought down to max_norm: the factor itself has no fp32 of full precision, the results have
    grads = []
    for i, n in enumerate(sizes):
        g = torch.Generator(device="cuda").manual_seed(i)
        size = 10.0 ** (30 + 8 * torch.rand(n, generator=g, device="cuda", dtype=torch.float64))
        grads.append((torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -1.0, 1.0) * size).to(dtype))
    kept = [g.clone() for g in grads]
    outs = None if place == "in place" else [torch.full_like(g, 9.0) for g in grads]
    lists = P.GradList(grads, outs)
    with P.Context(1, 8) as ctx:
        norm = ctx.clip_grad_norm(lists, max_norm)
        ctx.check()
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in kept))
    if want < 3e38:
        assert abs(float(norm) - want) <= 18 * U * want
    for o, g in zip(lists.out, kept):
        s = g.double() * (max_norm / want)
        # as for any other factor: 20 u, a rounding to the result's type; results below 2^-126 are multiples of 2^-149
        tol = (20 * U + (2.0 ** -8 if dtype == torch.bfloat16 else 0)) * s.abs() + (2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149)
        assert bool(((o.double() - s).abs() <= tol).all())


# ---- arguments that overlap --------------------------------------------------------------------------------------------------------
def test_rows_packed_over_themselves_and_margins_over_their_rows_are_refused(P, wpsgd_lib):
    lib, n, d = wpsgd_lib, 50, 100
    x = torch.randn(n, 128, device="cuda")
    q = torch.zeros(n, 512, dtype=torch.uint8, device="cuda")
    s, m, t = torch.zeros(n, 4, device="cuda"), torch.zeros(7, 112, dtype=torch.uint8, device="cuda"), torch.zeros(7, 1, device="cuda")
    z = torch.zeros(n, 7, device="cuda")
    with P.Context(1, d) as ctx:
        h = ctx._h

        def status(fn, *args):
            return fn(h, *[a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args])

        quant = lib.wpsgd_quantize_rows
        assert status(quant, x, 0, 128, n, x, 512, s, 4) == 1                           # codes over the rows
        assert status(quant, x, 0, 128, n, x.data_ptr() + 128 * 4 * (n - 1) + 16, 512, s, 4) == 1
        assert status(quant, x, 0, 128, n, q, 512, x, 128) == 1                         # scales over the rows
        assert status(quant, x, 0, 128, n, q, 512, q, 128) == 1                         # scales over the codes
        assert status(quant, x, 0, 128, n, x.data_ptr() + 400, 512, s, 4) == 0          # codes of the first rows in the padding of the rows
        marg = lib.wpsgd_margins_fp8
        for over in (q, m, s, t):
            assert status(marg, q, 512, s, 4, n, m, 112, t, 1, 7, over, 0, 7) == 1
        assert status(marg, q, 512, s, 4, n, m, 112, t, 1, 7, q.data_ptr() + 96, 1, 256) == 1
        assert lib.wpsgd_last_error(h) == b"margins_fp8: Z overlaps rows, models or their scales"
        assert status(marg, q, 512, s, 4, n, m, 112, t, 1, 7, z, 0, 7) == 0
        ctx.check()


def test_scales_and_margins_in_the_padding_of_the_packed_rows(P):
    # one buffer: 100 codes, 4 bytes of scale at 100, margins on 7 models from 112 on
    n, d, m = 300, 100, 7
    x, w = torch.randn(n, d, device="cuda"), torch.randn(m, d, device="cuda")
    buf = torch.full((n, 256), 0x55, dtype=torch.uint8, device="cuda")
    f = buf.view(torch.float32)
    with P.Context(1, d) as ctx:
        Q, S = ctx.quantize_rows(x)
        M, T = ctx.quantize_rows(w)
        ctx.quantize_rows(x, buf[:, :d], f[:, 25:26])
        z = ctx.margins_fp8(Q, S, M, T)
        ctx.margins_fp8(buf[:, :d], f[:, 25:26], M, T, out=f[:, 28:35])
        ctx.check()
    assert torch.equal(buf[:, :d], Q.view(torch.uint8)) and torch.equal(f[:, 25:26], S) and torch.equal(f[:, 28:35], z)
    assert bool((buf[:, 104:112] == 0x55).all()) and bool((buf[:, 140:] == 0x55).all())


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3", "two passes"])
@pytest.mark.parametrize("n", [40, 30000])
def test_gradient_written_over_the_rows_and_labels_it_was_made_from(P, kind, n):
    # everything is read before grad and out are written
    d = 8200 if kind == "two passes" else 200
    x, y, w = rows_problem(n, d)
    rows, _ = rows_of(kind, x)
    with P.Context(1, d) as ctx:
        fn = ctx.objective_grad_fp8 if kind == "e4m3" else ctx.objective_grad
        out, grad = fn(*rows, y, w, 0.01, 1)
        over = torch.as_strided(rows[0].view(torch.uint8) if kind == "e4m3" else rows[0], (4 * d // rows[0].element_size(),), (1,)).view(torch.float32)
        fn(*rows, y, w, 0.01, 1, grad=over, out=y[5:7])
        ctx.check()
    assert torch.equal(over, grad) and torch.equal(y[5:7], out)


def test_pointers_off_their_elements_are_refused(P, wpsgd_lib):
    # an access to them would end the process's use of the GPU: only ever run against a library that refuses
    lib, n, d = wpsgd_lib, 4, 100
    x = torch.zeros(n, d, device="cuda")
    q, s = torch.zeros(n, 112, dtype=torch.uint8, device="cuda"), torch.zeros(n + 1, 1, device="cuda")
    y, w, g, out = (torch.zeros(k + 1, device="cuda") for k in (n, d, d, 2))
    z = torch.zeros(n, n, device="cuda")
    with P.Context(1, d) as ctx:
        def refused(fn, *args, why=b"aligned to"):
            assert fn(ctx._h, *[a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args]) == 1
            assert why in lib.wpsgd_last_error(ctx._h)

        off = lambda t, by=2: t.data_ptr() + by
        refused(lib.wpsgd_quantize_rows, x, 0, d, n, q, 112, off(s), 1)
        refused(lib.wpsgd_margins_fp8, q, 112, off(s), 1, n, q, 112, s, 1, n, z, 0, n)
        refused(lib.wpsgd_margins_fp8, q, 112, s, 1, n, q, 112, off(s, 1), 1, n, z, 0, n)
        for i in range(4):
            at = [off(t, 1 + i % 3) if i == k else t for k, t in enumerate((y, w, g, out))]
            refused(lib.wpsgd_objective_grad, x, 0, d, at[0], n, at[1], 0.1, 0, at[2], at[3])
            refused(lib.wpsgd_objective_grad_fp8, q, 112, s, 1, at[0], n, at[1], 0.1, 0, at[2], at[3])
        refused(lib.wpsgd_objective_grad_fp8, q, 112, off(s), 1, y, n, w, 0.1, 0, g, out)
        lists = P.GradList([x])
        refused(lib.wpsgd_grad_norm, lists._h, off(out))
        refused(lib.wpsgd_clip_grad_norm, lists._h, 1.0, off(out))
        ctx.check()


def test_margins_and_packing_of_2_to_the_31_columns_are_refused(P, wpsgd_lib):
    # places in a tile are 32-bit coordinates: beyond, they would turn negative and read zeros. Nothing is read here
    lib, d = wpsgd_lib, 1 << 31
    q, s, z = torch.zeros(16, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    with P.Context(1, d) as ctx:
        assert lib.wpsgd_margins_fp8(ctx._h, q.data_ptr(), d, s.data_ptr(), d // 128, 1, q.data_ptr(), d, s.data_ptr(), d // 128, 1, z.data_ptr(), 0, 1) == 5
        assert lib.wpsgd_last_error(ctx._h).startswith(b"margins_fp8: 2^31 columns")
        assert lib.wpsgd_quantize_rows(ctx._h, z.data_ptr(), 0, d, 1, q.data_ptr(), d, s.data_ptr(), d // 128) == 5
        ctx.check()


# ---- a first call beside another stream's capture ---------------------------------------------------------------------------------
def test_a_first_call_while_another_stream_is_captured(P):
    # the workspace is allocated then, which must not end the capture (of another context, in CUDA's strictest mode)
    n, d = 300, 200
    x, y, w = rows_problem(n, d)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    grads, outs = [torch.zeros(d, device="cuda") for _ in sides], [torch.zeros(2, device="cuda") for _ in sides]
    a, b = (P.Context(1, d, stream=s) for s in sides)
    with torch.cuda.stream(sides[0]):
        want = a.objective_grad(x, y, w, 0.01, 1)
        sides[0].synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=sides[0], capture_error_mode="global"):
            a.objective_grad(x, y, w, 0.01, 1, grad=grads[0], out=outs[0])
            b.objective_grad(x, y, w, 0.01, 1, grad=grads[1], out=outs[1])
        graph.replay()
    a.check()
    b.check()
    for grad, out in zip(grads, outs):
        assert torch.equal(grad, want[1]) and torch.equal(out, want[0])
    del graph
    a.destroy()
    b.destroy()


@pytest.mark.parametrize("loss", [3, -1, 1 << 32, (1 << 32) + 1, -(1 << 32)])
def test_unknown_losses_are_refused(P, loss):
    x, y, w = rows_problem(4, 100)
    with P.Context(1, 100) as ctx:
        q, s = ctx.quantize_rows(x)
        for call in (lambda: ctx.objective_grad(x, y, w, 0.1, loss), lambda: ctx.objective_grad_fp8(q, s, y, w, 0.1, loss)):
            with pytest.raises(P.WpsgdError) as e:
                call()
            assert e.value.status_name == "INVALID_ARG"
        ctx.check()
