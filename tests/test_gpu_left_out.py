"""Rows that a call leaves out, through the public entry points: tensors that a call itself makes hold zeros there and nothing left over, models of chains that are
left out are those they started from, and rows outside every chain are not read. Everything here is exact."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


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


def leave_nans(*like):
    """Memory of these shapes given back full of NaN, enough of it that the next tensor of such a shape is made of it."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    made = [torch.full(shape, float("nan"), dtype=dtype, device="cuda") for shape, dtype in like for _ in range(40)]
    torch.cuda.synchronize()
    del made


def chain_rows(n, hk, hv, dk, dv, dtype, seed=0):
    g = gen(seed + n)
    q, k, v = (torch.randn(s, generator=g) for s in ((n, hk, dk), (n, hk, dk), (n, hv, dv)))
    q, k = (x / x.norm(dim=-1, keepdim=True).clamp_min(1e-6) for x in (q, k))
    decay = -torch.exp(torch.randn((n, hv), generator=g) - 2.0)
    return [x.to(dtype).cuda() for x in (q, k, v, decay, torch.sigmoid(torch.randn((n, hv), generator=g)))]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,top,d", [(1, 1, 8), (40, 2, 999), (300, 3, 64), (3001, 4, 1001), (2500, 2, 4096)])
def test_new_gradients_of_combine_are_zeros_where_no_place_is(ctx, dtype, n, top, d):
    node = torch.randint(0, 5, (n, top), generator=gen(n), dtype=torch.int32)
    node[torch.rand((n, top), generator=gen(1)) < 0.3] = -1
    node[0, 0] = -1
    where, _, off = ctx.sort_rows(node.cuda(), 5)
    y, dout = (torch.randn(s, generator=gen(i)).to(dtype).cuda() for i, s in enumerate([(n * top, d), (n, d)]))
    w = torch.rand((n, top), generator=gen(2)).cuda()
    want, want_w = ctx.combine_rows_grad(dout, y, where, w, torch.zeros_like(y))
    leave_nans((y.shape, dtype))
    dy, dw = ctx.combine_rows_grad(dout, y, where, w)
    ctx.check()
    assert int(off[-1]) < n * top and torch.equal(dy, want) and torch.equal(dw, want_w)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_sorted,d,pad,offset", [(1, 1, 0, 0), (33, 7, 1, 3), (100, 64, 0, 0), (4001, 2100, 0, 0), (4001, 2100, 5, 3), (2000, 5003, 2, 1), (1 << 21, 5, 0, 1), (700, 20000, 8, 8)])
def test_clear_rows(P, ctx, dtype, n_sorted, d, pad, offset):
    """Rows without a place are zeros after it, what lies between rows is as it was; few bytes and many, rows that start anywhere."""
    lib = P.load_library()
    flat = torch.full((offset + n_sorted * (d + pad) + 64,), 7.0, dtype=dtype, device="cuda")
    rows = flat[offset:offset + n_sorted * (d + pad)].view(n_sorted, d + pad)
    where = torch.randint(-1, n_sorted + 2, (n_sorted // 3 + 1, 2), generator=gen(d), dtype=torch.int32)
    where[0, 0], where[0, 1] = n_sorted - 1, 2 ** 31 - 1
    marks = torch.full(((n_sorted + 31) // 32,), -1, dtype=torch.int32, device="cuda")
    on = where.cuda()
    torch.cuda.synchronize()
    assert lib.wpsgd_clear_rows(ctx._h, on.data_ptr(), len(where), 2, rows.data_ptr(), int(dtype is torch.bfloat16), d + pad, d, n_sorted, marks.data_ptr()) == 0
    ctx.check()
    has = torch.zeros(n_sorted, dtype=torch.bool)
    has[where[(where >= 0) & (where < n_sorted)].long()] = True
    without = (~has).cuda()
    assert not bool(rows[without, :d].any()) and bool((rows[:, d:] == 7).all()) and bool((flat[:offset] == 7).all()) and bool((flat[offset + n_sorted * (d + pad):] == 7).all())
    if n_sorted * d * flat.element_size() > 16 << 20:
        assert bool((rows[~without, :d] == 7).all())  # many bytes: no other row is touched
    for args in ((None, len(where), 2, rows.data_ptr(), 0, d + pad, d, n_sorted, marks.data_ptr()), (on.data_ptr(), len(where), 2, rows.data_ptr(), 0, d + pad, d, n_sorted, None),
                 (on.data_ptr(), len(where), 2, rows.data_ptr(), 7, d + pad, d, n_sorted, marks.data_ptr()), (on.data_ptr(), len(where), 0, rows.data_ptr(), 0, d + pad, d, n_sorted, marks.data_ptr()),
                 (on.data_ptr(), len(where), 2, on.data_ptr(), 0, 1, 1, 1, marks.data_ptr()), (on.data_ptr(), len(where), 2, marks.data_ptr(), 0, 1, 1, 1, marks.data_ptr()),
                 (on.data_ptr(), len(where), 2, rows.data_ptr(), 0, d + pad, d, n_sorted, on.data_ptr())):
        assert lib.wpsgd_clear_rows(ctx._h, *args) == 1 and lib.wpsgd_last_error(ctx._h).startswith(b"clear_rows:")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,top,d", [(1, 1, 8), (40, 2, 999), (300, 3, 64), (3001, 4, 1001), (2500, 2, 4096)])
def test_new_rows_of_gather_are_zeros_where_no_place_is(ctx, dtype, n, top, d):
    node = torch.randint(0, 5, (n, top), generator=gen(n), dtype=torch.int32)
    node[torch.rand((n, top), generator=gen(1)) < 0.3] = -1
    node[0, 0] = -1
    where, _, off = ctx.sort_rows(node.cuda(), 5)
    x = torch.randn((n, d), generator=gen(3)).to(dtype).cuda()
    want = ctx.gather_rows(x, where, torch.zeros((n * top, d), dtype=dtype, device="cuda"))
    leave_nans(((n * top, d), dtype))
    got = ctx.gather_rows(x, where)
    ctx.check()
    assert int(off[-1]) < n * top and torch.equal(got, want)


LEFT = [  # lengths, first row, rows behind, heads_k, heads_v, dk, dv
    ([1, 1], 0, 1, 1, 1, 16, 16), ([0, 30, 65], 7, 200, 2, 4, 64, 32), ([100, 28], 300, 5, 2, 2, 60, 33), ([64], 1, 0, 1, 3, 128, 128), ([0, 0], 4, 90, 1, 2, 31, 70), ([], 0, 66, 1, 2, 24, 16),
    ([5] * 40, 3000, 3000, 1, 1, 128, 80),
]


@pytest.mark.parametrize("lengths,first,behind,hk,hv,dk,dv", LEFT)
def test_gradients_of_rows_outside_every_chain_are_zeros(ctx, lengths, first, behind, hk, hv, dk, dv):
    n, end = first + sum(lengths) + behind, first + sum(lengths)
    rows = chain_rows(n, hk, hv, dk, dv, torch.bfloat16)
    off = torch.tensor([first] + lengths).cumsum(0).cuda()
    dout = torch.randn((n, hv, dv), generator=gen(4)).to(torch.bfloat16).cuda()
    _, _, saved = ctx.delta_run(*rows, off, save=True)
    leave_nans(*[(x.shape, torch.bfloat16) for x in rows])
    got = ctx.delta_grad(saved, dout)[:5]
    ctx.check()
    few = [x[first:end].contiguous() for x in rows]  # the same rows without those around them
    want = ctx.delta_grad(ctx.delta_run(*few, off - first, save=True)[2], dout[first:end].contiguous())[:5] if end > first else [x[:0] for x in rows]
    for a, b in zip(got, want):
        assert torch.equal(a[first:end], b) and not bool(a[:first].any()) and not bool(a[end:].any())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths,first,behind,hk,hv,dk,dv", LEFT)
def test_new_answers_of_rows_outside_every_chain_are_zeros(ctx, lengths, first, behind, hk, hv, dk, dv, dtype):
    n, end = first + sum(lengths) + behind, first + sum(lengths)
    rows = chain_rows(n, hk, hv, dk, dv, dtype)
    off = torch.tensor([first] + lengths).cumsum(0).cuda()
    want = torch.full((n, hv, dv), 5.0, dtype=dtype, device="cuda")
    W = ctx.delta_run(*rows, off, out=want)[1]
    assert bool((want[:first] == 5).all()) and bool((want[end:] == 5).all())  # a tensor that is given keeps what it has there
    calls = [False, True] if dtype is torch.bfloat16 else [False]
    for save in calls:
        leave_nans((want.shape, dtype))
        got = ctx.delta_run(*rows, off, save=save)
        assert torch.equal(got[0][first:end], want[first:end]) and not bool(got[0][:first].any()) and not bool(got[0][end:].any()) and torch.equal(got[1], W)
    ctx.check()


@pytest.mark.parametrize("start", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
def test_chains_that_are_left_out_keep_their_models(P, dtype, start):
    rows = chain_rows(50, 1, 2, 16, 24, dtype)
    W0 = torch.randn((2, 2, 24, 16), generator=gen(1)).cuda() if start else None
    for off, good in (([0, 30, 20], 0), ([20, 10, 50], 1), ([0, 51, 52], None), ([-1, 20, 1 << 40], None)):
        with P.Context(1, 1) as c:
            out = torch.full((50, 2, 24), 7.0, dtype=dtype, device="cuda")
            leave_nans(((2, 2, 24, 16), torch.float32))
            _, W = c.delta_run(*rows, torch.tensor(off).cuda(), W0=W0, out=out)
            with pytest.raises(P.WpsgdError):
                c.check()
            want, answered = (torch.zeros_like(W) if W0 is None else W0.clone()), torch.zeros(50, dtype=torch.bool)
            if good is not None and dtype is torch.float32:  # row by row, chains whose offsets are in order run; in chunks none does
                part = slice(off[good], off[good + 1])
                answered[part] = True
                o, want[good:good + 1] = c.delta_run(*[x[part] for x in rows], torch.tensor([0, off[good + 1] - off[good]]).cuda(), W0=None if W0 is None else W0[good:good + 1])
                assert torch.equal(out[part], o)
            assert torch.equal(W, want) and bool((out[~answered] == 7).all())


class DeltaRows(ctypes.Structure):
    """wpsgd_delta_rows"""

    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "v", "g", "beta")] + [(n, ctypes.c_int64) for n in ("ld_q", "ld_k", "ld_v", "ld_g", "ld_beta")]
                + [("shard_off", ctypes.c_void_p), ("n_rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("n_chains", "heads_k", "heads_v", "dk", "dv")]
                + [("type", ctypes.c_int), ("scale", ctypes.c_float)])


def c_rows(rows, off, n_chains=None):
    q, k, v, g, beta = rows
    assert all(x.is_contiguous() for x in rows)
    return DeltaRows(*[x.data_ptr() for x in rows], *[x[0].numel() for x in rows], None if off is None else off.data_ptr(), len(q), len(off) - 1 if n_chains is None else n_chains, q.shape[1],
                     v.shape[1], q.shape[2], v.shape[2], int(q.dtype is torch.bfloat16), 0.5)


@pytest.mark.parametrize("first,end", [(70, 131), (0, 64), (200, 200)])
def test_rows_outside_every_chain_are_not_read(P, ctx, first, end):
    """Heads that are laid out anew: the workspaces hold the same, to the byte, whatever stands in rows outside the chains."""
    lib, n = P.load_library(), 200
    off = torch.tensor([first, first, end]).cuda()
    kept = []
    for other in (1.0, -2.0):
        rows = chain_rows(n, 2, 2, 60, 33, torch.bfloat16)
        dout = torch.randn((n, 2, 33), generator=gen(9)).to(torch.bfloat16).cuda()
        for x in rows + [dout]:
            x[:first] = other
            x[end:] = other
        r, size = c_rows(rows, off), ctypes.c_int64()
        spaces, outs = [], [torch.full_like(dout, 3.0)] + [torch.zeros_like(x) for x in rows]
        for use in (1, 2):
            assert lib.wpsgd_delta_workspace(ctypes.byref(r), use, ctypes.byref(size)) == 0
            spaces.append(torch.full((size.value,), 0x5A, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert lib.wpsgd_delta_run(ctx._h, ctypes.byref(r), None, None, outs[0].data_ptr(), 66, 1, spaces[0].data_ptr(), spaces[0].numel()) == 0
        assert lib.wpsgd_delta_grad(ctx._h, ctypes.byref(r), spaces[0].data_ptr(), spaces[0].numel(), dout.data_ptr(), 66, None, *[x.data_ptr() for x in outs[1:]], None, spaces[1].data_ptr(),
                                    spaces[1].numel()) == 0
        ctx.check()
        kept.append(spaces + outs)
    assert all(torch.equal(a, b) for a, b in zip(*kept))


def test_a_step_does_not_look_at_the_number_of_chains(P, ctx):
    lib = P.load_library()
    rows = chain_rows(6, 1, 2, 16, 8, torch.float32)
    W = torch.zeros((6, 2, 8, 16), device="cuda")
    want = ctx.delta_step(*rows, W.clone(), scale=0.5)
    for n_chains in (-1, 1 << 30, 0):
        r, out, mine = c_rows(rows, None, n_chains), torch.zeros_like(want), W.clone()
        torch.cuda.synchronize()
        assert lib.wpsgd_delta_step(ctx._h, ctypes.byref(r), mine.data_ptr(), None, 6, out.data_ptr(), 16) == 0
        ctx.check()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths,first,behind,hk,hv,dk,dv", LEFT)
@pytest.mark.parametrize("pad,by", [(0, 1), (5, 0), (8, 8)])
def test_new_answers_in_rows_further_apart(P, ctx, lengths, first, behind, hk, hv, dk, dv, pad, by, dtype):
    """WPSGD_DELTA_NEW_OUT on rows with a stride that start anywhere: zeros outside the chains, and what lies between the rows is as it was."""
    lib, n, width = P.load_library(), first + sum(lengths) + behind, hv * dv
    rows = chain_rows(n, hk, hv, dk, dv, dtype)
    off = torch.tensor([first] + lengths).cumsum(0).cuda()
    want = ctx.delta_run(*rows, off, scale=0.5)[0].flatten(1)
    r, size = c_rows(rows, off), ctypes.c_int64()
    assert lib.wpsgd_delta_workspace(ctypes.byref(r), 0, ctypes.byref(size)) == 0
    space = torch.zeros(size.value + 16, dtype=torch.uint8, device="cuda")
    flat = torch.full((by + n * (width + pad) + 8,), 7.0, dtype=dtype, device="cuda")
    out = flat[by:by + n * (width + pad)].view(n, width + pad)
    torch.cuda.synchronize()
    assert lib.wpsgd_delta_run(ctx._h, ctypes.byref(r), None, None, out.data_ptr(), width + pad, 4, space.data_ptr(), size.value) == 0
    ctx.check()
    assert torch.equal(out[:, :width], want) and bool((out[:, width:] == 7).all()) and bool((flat[:by] == 7).all()) and bool((flat[by + n * (width + pad):] == 7).all())
    for use in (2, 3, 6, 8, -1):
        assert lib.wpsgd_delta_run(ctx._h, ctypes.byref(r), None, None, out.data_ptr(), width + pad, use, space.data_ptr(), size.value) == 1


@pytest.mark.parametrize("n,d", [(200, 64), (3000, 2000)])
def test_replayed_with_other_places(P, d, n):
    """A graph's own tensors, few bytes and many: rows that lose their place between replays are zeros again."""
    top, k = 2, 7
    s = torch.cuda.Stream()
    x, w = torch.randn((n, d), generator=gen(1)).cuda(), torch.rand((n, top), generator=gen(2)).cuda()
    nodes = []
    for seed, dropped in ((3, 0.0), (4, 0.6), (5, 0.2)):
        node = torch.randint(0, k, (n, top), generator=gen(seed), dtype=torch.int32)
        node[torch.rand((n, top), generator=gen(seed + 10)) < dropped] = -1
        nodes.append(node.cuda())
    at = nodes[0].clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(s), P.Context(k, d, stream=s) as c:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            where, _, off = c.sort_rows(at)
            rows = c.gather_rows(x, where)
            dy, dw = c.combine_rows_grad(x, rows, where, w)
        for node in nodes:
            at.copy_(node)
            graph.replay()
            want_where, _, want_off = c.sort_rows(node)
            want = c.gather_rows(x, want_where, torch.zeros_like(rows))
            want_dy, want_dw = c.combine_rows_grad(x, want, want_where, w, torch.zeros_like(rows))
            s.synchronize()
            assert torch.equal(where, want_where) and torch.equal(rows, want) and torch.equal(dy, want_dy) and torch.equal(dw, want_dw)
        c.check()
        graph.reset()
