"""Rows sorted by node, laid out in that order and brought back with weights, through the public entry points, against plain statements of
the same. Sorting and copying are exact; tolerances of sums count roundings (u = 2^-24 in fp32, half a step of the result's type)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def P(wpsgd_lib):
    import paper_1708_04801_b200 as pkg

    return pkg


@pytest.fixture(scope="module")
def ctx(P):
    with P.Context(16, 8) as c:
        yield c
        c.check()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def assignment(n, top, nodes, seed, dropped=0.2):
    node = torch.randint(0, nodes, (n, top), generator=gen(seed), dtype=torch.int32)
    node[torch.rand((n, top), generator=gen(seed + 1)) < dropped] = -1
    return node


def sorted_reference(node, nodes):
    """(where, order, shard_off), place by place."""
    flat = node.reshape(-1).tolist()
    places = [e for k in range(nodes) for e in [i for i, x in enumerate(flat) if x == k]] if len(flat) < 3000 else \
        [e for _, e in sorted((x, i) for i, x in enumerate(flat) if x >= 0)]
    where, order = [-1] * len(flat), [-1] * len(flat)
    for pos, e in enumerate(places):
        where[e], order[pos] = pos, e
    counts = torch.bincount(node.reshape(-1)[node.reshape(-1) >= 0].long(), minlength=nodes)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    return torch.tensor(where, dtype=torch.int32).view(node.shape), torch.tensor(order, dtype=torch.int32), off


def strided(t, pad, offset=0, fill=77.0):
    """The same values on the GPU in rows `pad` elements further apart, the first `offset` elements into its storage."""
    n, d = t.shape
    flat = torch.full((offset + n * (d + pad),), fill).to(t.dtype).cuda()
    v = flat[offset:].view(n, d + pad)[:, :d]
    v.copy_(t)
    return v


# ---- sorting ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,top,nodes,dropped", [
    (1, 1, 1, 0.0), (1, 1, 5, 1.0), (0, 3, 7, 0.0), (7, 3, 4, 0.3), (31, 1, 2, 0.0), (64, 2, 16, 0.0), (333, 3, 1000, 0.2), (4096, 1, 3, 0.0),
    (4097, 1, 1, 0.1), (5000, 2, 128, 0.0), (9000, 2, 37, 0.5), (40001, 2, 1025, 0.1), (70000, 2, 16384, 0.0), (300, 2, 16384, 0.1), (50001, 8, 129, 0.02),
    (32768, 1, 64, 0.0), (33000, 1, 1300, 0.9), (100003, 3, 2, 0.3), (40000, 5, 2048, 0.0), (300000, 2, 100, 1.0), (65536, 1, 5461, 0.0), (1 << 20, 2, 64, 0.01),
])
def test_sort_rows(ctx, n, top, nodes, dropped):
    node = assignment(n, top, nodes, n + nodes, dropped)
    where, order, off = ctx.sort_rows(node.cuda(), nodes)
    want = sorted_reference(node, nodes)
    ctx.check()
    assert torch.equal(off.cpu(), want[2]) and torch.equal(where.cpu(), want[0]) and torch.equal(order.cpu(), want[1])


def test_sort_rows_one_node_has_everything(ctx):
    node = torch.full((20000, 4), 9, dtype=torch.int32)
    where, order, off = ctx.sort_rows(node.cuda())
    assert torch.equal(where.cpu().view(-1), torch.arange(80000, dtype=torch.int32)) and torch.equal(order.cpu(), torch.arange(80000, dtype=torch.int32))
    assert off.tolist() == [0] * 10 + [80000] * 7


def test_nodes_and_positions_past_the_end_count_as_none_and_are_reported(P):
    with P.Context(4, 8) as c:
        node = torch.tensor([[0, 4], [3, 2147483647], [-2147483648, 1]], dtype=torch.int32).cuda()
        where, order, off = c.sort_rows(node)
        assert where.tolist() == [[0, -1], [2, -1], [-1, 1]] and off.tolist() == [0, 1, 2, 2, 3] and order.tolist() == [0, 5, 2, -1, -1, -1]
        with pytest.raises(P.WpsgdError):
            c.check()
    y = torch.ones(3, 8).cuda()
    at = torch.tensor([[0, 3], [2147483647, 2]], dtype=torch.int32).cuda()
    for call in (lambda c: c.combine_rows(y, at), lambda c: c.combine_rows_grad(y[:2], y, at)[1], lambda c: c.gather_rows(y[:2], at, torch.zeros(3, 8).cuda())):
        with P.Context(4, 8) as c:
            got = call(c)
            if got.shape == (2, 8):
                assert bool((got == 1).all())
            elif got.shape == (2, 2):
                assert got.tolist() == [[8.0, 0.0], [0.0, 8.0]]
            else:
                assert got.sum(1).tolist() == [8.0, 0.0, 8.0]
            with pytest.raises(P.WpsgdError):
                c.check()


# ---- rows there and back -----------------------------------------------------------------------------------------------------
SHAPES = [  # rows, top, d, padding and offset in elements
    (1, 1, 1, 0, 0), (5, 3, 7, 0, 0), (64, 2, 1024, 0, 0), (33, 5, 999, 0, 0), (33, 2, 999, 1, 0), (20, 9, 130, 0, 3), (300, 1, 64, 8, 8), (9, 2, 8192, 0, 0),
    (7, 4, 8191, 0, 1), (2500, 2, 40, 0, 0), (3, 2, 20000, 0, 0), (65, 3, 8, 4, 4), (17, 2, 12, 0, 5),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,top,d,pad,offset", SHAPES)
def test_gather_rows(ctx, dtype, n, top, d, pad, offset):
    x = torch.randn((n, d), generator=gen(d)).to(dtype)
    node = assignment(n, top, 11, n)
    where, order, off = ctx.sort_rows(node.cuda(), 11)
    to = strided(torch.full((n * top, d), 5.0).to(dtype), pad, (offset * 3) % 16)
    before = to.clone()
    got = ctx.gather_rows(strided(x, pad, offset, float("nan")), where, to)
    ctx.check()
    kept = int(off[-1])
    want = x[order[:kept].cpu().long() // top]
    assert got is to and torch.equal(got[:kept].cpu(), want) and torch.equal(got[kept:], before[kept:])
    if pad:
        assert bool((to.as_strided((n * top - 1, pad), (d + pad, 1), to.storage_offset() + d) == 77.0).all())


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,top,d,pad,offset", SHAPES)
def test_combine_rows(ctx, dtype, n, top, d, pad, offset, weighted):
    node = assignment(n, top, 11, n)
    where, _, _ = sorted_reference(node, 11)
    y = torch.randn((n * top, d), generator=gen(d)).to(dtype)
    y[int((node >= 0).sum()):] = float("nan")         # rows that no place has
    w = torch.randn((n, top), generator=gen(1))
    w[node < 0] = float("inf")                          # a place without a row has no weight
    to = strided(torch.full((n, d), 5.0).to(dtype), pad, (offset * 5) % 16)
    got = ctx.combine_rows(strided(y, pad, offset, float("nan")), where.cuda(), w.cuda() if weighted else None, to)
    ctx.check()
    used = torch.where(node < 0, torch.zeros(()), w if weighted else torch.ones(())).double()
    rows = torch.where((where < 0)[..., None], torch.zeros((), dtype=torch.float64), y[where.clamp_min(0).long()].double())
    want, size = (used[..., None] * rows).sum(1), (used[..., None] * rows).abs().sum(1)
    # top products and sums in fp32, one rounding to the type
    bound = top * U * size + (torch.finfo(dtype).eps / 2) * (want.abs() + top * U * size) + 1e-38
    assert bool(((got.cpu().double() - want).abs() <= bound).all())
    if pad and n > 1:
        assert bool((to.as_strided((n - 1, pad), (d + pad, 1), to.storage_offset() + d) == 77.0).all())


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,top,d,pad,offset", SHAPES)
def test_combine_rows_grad(ctx, dtype, n, top, d, pad, offset, weighted):
    node = assignment(n, top, 11, n)
    where, order, off = sorted_reference(node, 11)
    kept = int(off[-1])
    y = torch.randn((n * top, d), generator=gen(d)).to(dtype)
    y[kept:] = float("nan")
    dout = torch.randn((n, d), generator=gen(d + 1)).to(dtype)
    w = torch.randn((n, top), generator=gen(1))
    to = strided(torch.full((n * top, d), 5.0).to(dtype), pad, (offset * 7) % 16)
    dy, dw = ctx.combine_rows_grad(strided(dout, pad, offset, float("nan")), strided(y, 0, 0), where.cuda(), w.cuda() if weighted else None, to)
    ctx.check()
    place = order[:kept].long()
    used = (w if weighted else torch.ones_like(w)).view(-1)[place]
    want = (used[:, None] * dout[place // top].float()).to(dtype)     # one product in fp32, rounded once: the same on both sides
    assert torch.equal(dy[:kept].cpu(), want) and bool((dy[kept:] == 5.0).all())
    there = where >= 0
    products = dout.double()[:, None] * torch.where(there[..., None], y[where.clamp_min(0).long()].double(), torch.zeros((), dtype=torch.float64))
    assert bool(((dw.cpu().double() - products.sum(2)).abs() <= d * U * products.abs().sum(2)).all())
    assert bool((dw.cpu()[~there] == 0).all())


def test_gradients_are_those_of_differences(ctx):
    n, top, d = 6, 2, 5
    node = assignment(n, top, 3, 5)
    where = ctx.sort_rows(node.cuda(), 3)[0]
    y, w, dout = (torch.randn(s, generator=gen(i)).cuda() for i, s in enumerate([(n * top, d), (n, top), (n, d)]))
    dy, dw = ctx.combine_rows_grad(dout, y, where, w, torch.zeros_like(y))
    value = lambda a, b: float((ctx.combine_rows(a, where, b).double() * dout.double()).sum())  # noqa: E731
    h = 2.0 ** -4  # the result is linear in each: differences are exact but for roundings, of which the sums have about 2^-20
    for i in range(n * top):
        e = torch.zeros_like(y)
        e[i, i % d] = h
        assert abs((value(y + e, w) - value(y - e, w)) / (2 * h) - float(dy[i, i % d])) < 1e-4
    for i in range(n):
        e = torch.zeros_like(w)
        e[i, i % top] = h
        assert abs((value(y, w + e) - value(y, w - e)) / (2 * h) - float(dw[i, i % top])) < 1e-4


def test_gradient_of_gather_is_combine_without_weights(ctx):
    node = assignment(100, 3, 8, 2)
    where, order, off = ctx.sort_rows(node.cuda(), 8)
    g = torch.randn((300, 24), generator=gen(3))
    got = ctx.combine_rows(g.cuda(), where).cpu()
    want = torch.zeros(100, 24, dtype=torch.float64)
    kept = int(off[-1])
    want.index_add_(0, order[:kept].cpu().long() // 3, g[:kept].double())
    assert bool(((got.double() - want).abs() <= 3 * U * 3 * g.abs().max()).all())


def test_large_rows_past_32_bits(ctx):
    # offsets of 2^31 bytes and more: the last rows of 5 GB
    n, d = 1 << 17, 20480
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn((3, d), generator=gen(1)).to(torch.bfloat16).cuda()
    at = torch.tensor([[n - 1], [n - 3], [n - 2]], dtype=torch.int32).cuda()
    assert torch.equal(ctx.combine_rows(x, at), x[[n - 1, n - 3, n - 2]])
    ctx.gather_rows(x[-3:], at - 1000, x[:n - 4])
    assert torch.equal(x[[n - 1001, n - 1003, n - 1002]], x[-3:])
    ctx.check()


def test_on_another_stream_and_in_a_graph(P):
    node = assignment(500, 2, 16, 7)
    want = sorted_reference(node, 16)
    x = torch.randn((500, 96), generator=gen(8)).cuda()
    w = torch.rand((500, 2), generator=gen(9)).cuda()
    s = torch.cuda.Stream()
    node_d = torch.zeros_like(node, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s), P.Context(16, 96, stream=s) as c:
        c.sort_rows(node_d)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            where, order, off = c.sort_rows(node_d)
            rows = torch.zeros(1000, 96, device="cuda")
            c.gather_rows(x, where, rows)
            back = c.combine_rows(rows, where, w)
            dy, dw = c.combine_rows_grad(x, rows, where, w, torch.zeros_like(rows))
        node_d.copy_(node)
        graph.replay()
        s.synchronize()
        assert torch.equal(where.cpu(), want[0]) and torch.equal(off.cpu(), want[2])
        used = torch.where(node < 0, torch.zeros(()), w.cpu()).double().sum(1, keepdim=True)
        assert bool(((back.cpu().double() - used * x.cpu().double()).abs() <= 4 * U * x.cpu().abs() * used.abs() + 1e-30).all())
        norms = (x.cpu().double() ** 2).sum(1)
        assert bool(((dw.cpu().double() - torch.where(node < 0, torch.zeros((), dtype=torch.float64), norms[:, None])).abs() <= 96 * U * norms[:, None]).all())
        c.check()
        graph.reset()


def test_refusals(P, ctx):
    x = torch.zeros(4, 8).cuda()
    at = torch.zeros(4, 2, dtype=torch.int32).cuda()
    for call in (lambda: ctx.sort_rows(at.long()), lambda: ctx.sort_rows(at.t()), lambda: ctx.sort_rows(at.cpu()), lambda: ctx.gather_rows(x.half(), at), lambda: ctx.gather_rows(x, at, x.bfloat16()),
                 lambda: ctx.combine_rows(x, at, torch.zeros(4, 2, dtype=torch.float64).cuda()), lambda: ctx.combine_rows(x, at.view(-1))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ctx.gather_rows(x[:3], at), lambda: ctx.gather_rows(x.t(), at), lambda: ctx.combine_rows(x, at, torch.zeros(4, 3).cuda()), lambda: ctx.combine_rows(x, at, None, x[:3]),
                 lambda: ctx.combine_rows_grad(x[:2], x, at), lambda: ctx.combine_rows_grad(x, x, at, None, torch.zeros(3, 8).cuda()), lambda: ctx.sort_rows(at, 1 << 40)):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: ctx.sort_rows(at, 16385), "UNSUPPORTED"), (lambda: ctx.sort_rows(at, 0), "INVALID_ARG"), (lambda: ctx.gather_rows(x, at, x), "INVALID_ARG"),
                         (lambda: ctx.combine_rows(x, at, None, x), "INVALID_ARG"), (lambda: ctx.combine_rows_grad(x, x, at, None, x), "INVALID_ARG"),
                         (lambda: ctx.combine_rows(x, torch.zeros(4, 0, dtype=torch.int32).cuda()), "INVALID_ARG")):
        with pytest.raises(P.WpsgdError) as e:
            call()
        assert e.value.status_name == status
