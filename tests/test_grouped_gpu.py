"""Products of rows sorted by expert with each expert's NVFP4 weights, and their gradients, against 64-bit products of the
values they hold."""
import pytest
import torch

import plain64
import workloads

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


def gen(*key):
    return workloads.generator(DEV, 601, *key)


def rand(shape, g, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def weights(experts, n, k, block, g):
    """Random nibbles, scale codes of every exponent, and a global scale for each expert."""
    q = torch.randint(0, 256, (experts, n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(0, 127, (experts, n, k // block), generator=g, device=DEV, dtype=torch.uint8)
    return q, sc, torch.rand((experts,), generator=g, device=DEV) + 0.01


def offsets_of(sizes, first=0):
    ends = [first]
    for s in sizes:
        ends.append(ends[-1] + s)
    return torch.tensor(ends, dtype=torch.int32, device=DEV)


def expected(rows, bounds, w, block, turned):
    """(values, bounds) of rows times each group's weights; zero outside; bounds: (first, end) of each group."""
    q, sc, S = w
    outer = q.shape[2] * 2 if turned else q.shape[1]
    want = torch.zeros((rows.shape[0], outer), dtype=torch.float64)
    lim = torch.zeros_like(want)
    for e, (a, b) in enumerate(bounds):
        if a >= b:
            continue
        v, s = plain64.nvfp4_values(q[e], sc[e], block), float(S[e])
        y, bound = plain64.product(plain64.f64(rows[a:b]), v.t() if turned else v)
        want[a:b] = y * s
        # the sum's product with the global scale is rounded once, before the output's own rounding
        lim[a:b] = bound * s + 2.0 ** -24 * (y.abs() + bound) * s
    return want, lim


def spans(offsets):
    o = offsets.tolist()
    return list(zip(o[:-1], o[1:]))


def both(nv, sizes, n, k, block, out, key, spare=0, first=0):
    g = gen(key, n, k, block)
    w = weights(len(sizes), n, k, block, g)
    rows = first + sum(sizes) + spare
    offsets = offsets_of(sizes, first)
    x, dy = rand((rows, k), g), rand((rows, n), g)
    want, lim = expected(x, spans(offsets), w, block, False)
    plain64.check(nv.grouped_matmul(x, offsets, *w, block=block, out_dtype=out), want, lim, "y")
    want, lim = expected(dy, spans(offsets), w, block, True)
    plain64.check(nv.grouped_matmul_grad_input(dy, offsets, *w, block=block, out_dtype=out), want, lim, "dx")


SIZES = {
    "one": [1], "ones": [1, 1, 0, 1], "empty ends": [0, 0, 3, 0, 16, 0], "few": [5, 17, 1, 0, 16], "some": [33, 31, 64, 20, 0],
    "ragged": [1, 130, 0, 257, 64, 3], "tall": [300, 129], "one of many": [0] * 70 + [40] + [0] * 60,
}


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,k", [(77, 208), (256, 512), (1, 16)])
@pytest.mark.parametrize("sizes", SIZES)
def test_sizes(nv, sizes, n, k, out):
    both(nv, SIZES[sizes], n, k, 16, out, 1)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("sizes,n,k", [([7, 0, 12], 130, 1152), ([30, 20], 96, 2176), ([150, 10, 90], 130, 640)])
def test_blocks(nv, sizes, n, k, block):
    both(nv, sizes, n, k, block, torch.bfloat16, 2)


# every number of weight rows of a workgroup for few rows, by the outputs that there are; k of no whole 32 too
@pytest.mark.parametrize("k", [272, 4096])
@pytest.mark.parametrize("each", [4, 24])
@pytest.mark.parametrize("n", [40, 1030, 4200])
def test_few_rows_widths(nv, n, each, k):
    both(nv, [each, 0, each + 3, 1] * 4, n, k, 16, torch.bfloat16, 3)


# the largest tile: its heights of 64, 128 and 256 rows, ends inside each; contractions of an odd number of steps
@pytest.mark.parametrize("n,k,out", [(8200, 64, torch.bfloat16), (8201, 80, torch.float32)])
def test_largest_tiles_forward(nv, n, k, out):
    g = gen(4, n)
    sizes = [300, 600, 513, 40, 380, 0, 256]
    w = weights(len(sizes), n, k, 16, g)
    offsets = offsets_of(sizes)
    x = rand((sum(sizes), k), g)
    want, lim = expected(x, spans(offsets), w, 16, False)
    plain64.check(nv.grouped_matmul(x, offsets, *w, out_dtype=out), want, lim, "y")


@pytest.mark.parametrize("n,k,out", [(64, 8208, torch.bfloat16), (203, 8192, torch.float32)])
def test_largest_tiles_gradient(nv, n, k, out):
    g = gen(5, n)
    sizes = [300, 600, 513, 40, 380, 0, 256]
    w = weights(len(sizes), n, k, 16, g)
    offsets = offsets_of(sizes)
    dy = rand((sum(sizes), n), g)
    want, lim = expected(dy, spans(offsets), w, 16, True)
    plain64.check(nv.grouped_matmul_grad_input(dy, offsets, *w, out_dtype=out), want, lim, "dx")


@pytest.mark.parametrize("each", [3, 25, 100])
def test_rows_of_no_expert(nv, each):
    """Zero in a new output, left as they were in one's own; what they hold does not matter."""
    g = gen(6, each)
    n, k, sizes = 90, 272, [each, 0, each + 1]
    w = weights(3, n, k, 16, g)
    offsets = offsets_of(sizes, 9)
    rows = 9 + sum(sizes) + 50
    inside = slice(9, 9 + sum(sizes))
    x, dy = rand((rows, k), g), rand((rows, n), g)
    for a in (x, dy):
        a[:9], a[9 + sum(sizes):] = float("nan"), float("inf")
    for f, a, turned in ((nv.grouped_matmul, x, False), (nv.grouped_matmul_grad_input, dy, True)):
        want, lim = expected(a, spans(offsets), w, 16, turned)
        got = f(a, offsets, *w)
        plain64.check(got, want, lim, "y")
        own = torch.full_like(got, 7.0)
        assert f(a, offsets, *w, out=own) is own
        assert torch.equal(own[inside], got[inside])
        assert bool((own[:9] == 7).all()) and bool((own[9 + sum(sizes):] == 7).all())


@pytest.mark.parametrize("each", [3, 25, 100])
def test_offsets_out_of_order_or_range(nv, each):
    """Offsets count as the nearest within the rows and never descend: nothing else is read or written."""
    g = gen(7, each)
    n, k, rows = 40, 64, 3 * each
    w = weights(4, n, k, 16, g)
    x = rand((rows, k), g)
    offsets = torch.tensor([-5, 2 * each, each, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    want, lim = expected(x, [(0, 2 * each), (0, 0), (2 * each, rows), (0, 0)], w, 16, False)
    plain64.check(nv.grouped_matmul(x, offsets, *w), want, lim, "y")
    none = torch.tensor([rows + 4] * 5, dtype=torch.int32, device=DEV)
    assert not nv.grouped_matmul(x, none, *w).any()


def test_many_experts(nv):
    """More experts than a wave takes at once, most without rows."""
    g = gen(8)
    sizes = [0] * 200
    for e, s in ((0, 2), (63, 5), (64, 70), (127, 1), (128, 3), (199, 300)):
        sizes[e] = s
    both(nv, sizes, 48, 96, 16, torch.float32, 8, spare=3)


@pytest.mark.parametrize("sizes", [[4, 0, 9], [28, 32], [200, 70]])
def test_rows_between_nans(nv, sizes):
    g = gen(9, len(sizes))
    n, k, rows = 90, 272, sum(sizes)
    w = weights(len(sizes), n, k, 16, g)
    offsets = offsets_of(sizes)
    x = rand((rows, k), g)
    assert torch.equal(nv.grouped_matmul(x, offsets, *w), nv.grouped_matmul(plain64.between_nans(x), offsets, *w))
    for width in (90, 88):
        dy = rand((rows, width), g)
        args = (offsets, w[0][:, :width].contiguous(), w[1][:, :width].contiguous(), w[2])
        assert torch.equal(nv.grouped_matmul_grad_input(dy, *args),
                           nv.grouped_matmul_grad_input(plain64.between_nans(dy), *args))


@pytest.mark.parametrize("each", [3, 25, 150])
def test_nan_and_infinity_stay_in_their_row(nv, each):
    g = gen(10, each)
    n, k = 50, 160
    w = weights(2, n, k, 16, g)
    offsets = offsets_of([each, each])
    x = rand((2 * each, k), g)
    clean = nv.grouped_matmul(x, offsets, *w)
    x[each, 3], x[1, 7] = float("nan"), float("inf")
    got = nv.grouped_matmul(x, offsets, *w)
    assert bool(got[each].isnan().all()) and not bool(got[1].isfinite().any())
    keep = [i for i in range(2 * each) if i not in (1, each)]
    assert torch.equal(got[keep], clean[keep])


def test_as_single_products(nv):
    """Each group as matmul() gives it for its rows, within both sums' bounds; one group alone is one product."""
    g = gen(11)
    n, k = 96, 512
    w = weights(3, n, k, 16, g)
    sizes = [6, 200, 40]
    offsets = offsets_of(sizes)
    x = rand((246, k), g)
    got = nv.grouped_matmul(x, offsets, *w, out_dtype=torch.float32)
    want, lim = expected(x, spans(offsets), w, 16, False)
    for e, (a, b) in enumerate(spans(offsets)):
        one = nv.matmul(x[a:b], w[0][e], w[1][e], w[2][e:e + 1], out_dtype=torch.float32)
        assert bool(((plain64.f64(one) - plain64.f64(got[a:b])).abs()
                     <= 2 * (lim[a:b] + 2.0 ** -24 * (want[a:b].abs() + lim[a:b]))).all())


@pytest.mark.parametrize("rows,experts,n,k", [(0, 3, 32, 64), (8, 3, 0, 64), (8, 3, 32, 0), (8, 0, 32, 64)])
def test_empty(nv, rows, experts, n, k):
    w = weights(experts, n, k, 16, gen(12))
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = rows
    x, dy = (torch.ones((rows, c), dtype=torch.bfloat16, device=DEV) for c in (k, n))
    y, dx = nv.grouped_matmul(x, offsets, *w), nv.grouped_matmul_grad_input(dy, offsets, *w)
    assert y.shape == (rows, n) and dx.shape == (rows, k)
    if k == 0 or experts == 0:
        assert not y.any()
    if n == 0 or experts == 0:
        assert not dx.any()


@pytest.mark.parametrize("each", [3, 25, 150])
def test_other_stream_and_repeats(nv, each):
    g = gen(13, each)
    n, k = 200, 2048
    w = weights(3, n, k, 16, g)
    offsets = offsets_of([each, 1, each])
    x, dy = rand((2 * each + 1, k), g), rand((2 * each + 1, n), g)
    want, want_dx = nv.grouped_matmul(x, offsets, *w), nv.grouped_matmul_grad_input(dy, offsets, *w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        later = x * 1
        for _ in range(20):
            later = later * 1
        got, got_dx = nv.grouped_matmul(later, offsets, *w), nv.grouped_matmul_grad_input(dy, offsets, *w)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(got_dx, want_dx)


@pytest.mark.parametrize("each", [4, 150])
def test_captured_and_replayed_with_other_offsets(nv, each):
    """A graph reads the offsets when it runs; eager work and synchronizations between the replays."""
    g = gen(14, each)
    n, k, rows = 72, 320, 4 * each
    w = weights(4, n, k, 16, g)
    x, dy = rand((rows, k), g), rand((rows, n), g)
    offsets = offsets_of([each] * 4)
    y, dx = torch.empty((rows, n), dtype=torch.bfloat16, device=DEV), torch.empty((rows, k), dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        nv.grouped_matmul(x, offsets, *w, out=y)
        nv.grouped_matmul_grad_input(dy, offsets, *w, out=dx)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nv.grouped_matmul(x, offsets, *w, out=y)
        nv.grouped_matmul_grad_input(dy, offsets, *w, out=dx)
    for sizes in ([each] * 4, [0, 3 * each, 1, each - 1], [1, 0, 0, 4 * each - 1], [4 * each, 0, 0, 0]):
        offsets.copy_(offsets_of(sizes))
        x.copy_(rand((rows, k), g))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, nv.grouped_matmul(x, offsets, *w))
        assert torch.equal(dx, nv.grouped_matmul_grad_input(dy, offsets, *w))


def test_autograd(nv):
    g = gen(15)
    n, k, sizes = 64, 128, [5, 0, 40, 3]
    w = weights(4, n, k, 16, g)
    offsets = offsets_of(sizes)
    x = rand((50, k), g).requires_grad_()                  # two rows behind the last expert's
    y = nv.grouped_matmul(x, offsets, *w)
    dy = rand((n, 50), g).t()                              # strided, as autograd may hand it over
    y.backward(dy)
    want, lim = expected(dy.contiguous(), spans(offsets), w, 16, True)
    plain64.check(x.grad, want, lim, "dx")
    assert not x.grad[48:].any() and not y[48:].any()
    with torch.no_grad():
        assert not nv.grouped_matmul(x, offsets, *w).requires_grad


def test_gradient_by_differences(nv):
    """The product is linear in x, so differences are exact but for the sums' roundings."""
    g = gen(16)
    n, k, sizes = 96, 128, [20, 13]
    w = weights(2, n, k, 16, g)
    offsets = offsets_of(sizes)
    x, dy = rand((33, k), g), rand((33, n), g)
    dx = plain64.f64(nv.grouped_matmul_grad_input(dy, offsets, *w, out_dtype=torch.float32))
    y0 = plain64.f64(nv.grouped_matmul(x, offsets, *w, out_dtype=torch.float32))
    for i, j in ((0, 0), (7, 31), (20, 5), (32, 127)):
        e = int(i >= 20)
        x1 = x.clone()
        x1[i, j] = x[i, j] + 4.0
        step = plain64.f64(x1)[i, j] - plain64.f64(x)[i, j]
        y1 = plain64.f64(nv.grouped_matmul(x1, offsets, *w, out_dtype=torch.float32))
        diff = ((y1 - y0) * plain64.f64(dy)).sum() / step
        v = plain64.nvfp4_values(w[0][e], w[1][e], 16) * float(w[2][e])
        noise = 2 * (k + 4) * plain64.SUM * ((plain64.f64(x1).abs() + plain64.f64(x).abs())[i] @ v.t().abs()
                                             * plain64.f64(dy).abs()[i]).sum() / step.abs()
        noise += (n + 4) * plain64.SUM * (plain64.f64(dy).abs()[i] @ v.abs())[j]
        assert abs(diff - dx[i, j]) <= noise


def test_long_offsets(nv):
    """The last rows of activations, and the last expert's weights, behind more than 2^32 bytes."""
    g = gen(17)
    k, rows = 8192, 2 ** 18 + 300
    x = torch.zeros((rows, k), dtype=torch.bfloat16, device=DEV)
    tail = rand((300, k), g)
    x[-300:] = tail
    w = weights(2, 48, k, 16, g)
    offsets = offsets_of([rows - 300, 300])
    y = nv.grouped_matmul(x, offsets, *w)
    want, lim = expected(tail, [(0, 0), (0, 300)], w, 16, False)
    plain64.check(y[-300:], want, lim, "y")
    assert not bool(y[:-300].any())
    del x, y
    experts, n = 70, 16384
    q = torch.zeros((experts, n, k // 2), dtype=torch.uint8, device=DEV)
    sc = torch.zeros((experts, n, k // 128), dtype=torch.uint8, device=DEV)
    last = weights(1, n, k, 128, g)
    q[-1], sc[-1] = last[0][0], last[1][0]
    S = torch.ones(experts, device=DEV)
    S[-1] = last[2][0]
    for rows in (5, 40):
        offsets = offsets_of([0] * (experts - 1) + [rows])
        x, dy = rand((rows, k), g), rand((rows, n), g)
        y = nv.grouped_matmul(x, offsets, q, sc, S, block=128)
        want, lim = expected(x, [(0, rows)], [t[:, -100:] if t.dim() > 1 else t for t in last], 128, False)
        plain64.check(y[:, -100:], want, lim, "y")
        one = [t[..., :] for t in last]
        dx = nv.grouped_matmul_grad_input(dy, offsets, q, sc, S, block=128, out_dtype=torch.float32)
        v = plain64.nvfp4_values(one[0][0][:, :64].contiguous(), one[1][0][:, :1].contiguous(), 128)
        want, bound = plain64.product(plain64.f64(dy), v.t())
        s = float(last[2][0])
        plain64.check(dx[:, :128], want * s, bound * s + 2.0 ** -24 * (want.abs() + bound) * s, "dx")


def xcd_runs(sizes, outer, height=256, width=256):
    """Tiles of each of the eight XCDs' runs, as the kernel deals them out."""
    count = sum(-(-s // height) for s in sizes) * -(-outer // width)
    return [count // 8 + (x < count % 8) for x in range(8)]


# one, two, four and three quarters of 32 compute units' worth of tiles over: cut into four, four, two parts, and whole
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("extra,over", [(1, 8), (0, 0), (2, 16), (3, 24)])
def test_last_tiles_in_parts(nv, extra, over, turned):
    g = gen(18, extra, turned)
    outer, inner = 16384, 64                               # 64 tiles across
    sizes = [700, 0, 256 + 1, 260, 200, 300, 256, 40][:6] + [256] * (extra + 2)
    tiles = sum(-(-s // 256) for s in sizes)
    while tiles % 4 != extra:
        sizes.append(130)
        tiles += 1
    assert set(r % 32 for r in xcd_runs(sizes, outer)) == {over}
    n, k = (inner, outer) if turned else (outer, inner)
    w = weights(len(sizes), n, k, 16, g)
    offsets = offsets_of(sizes, 3)
    x = rand((sum(sizes) + 10, inner), g)
    f = nv.grouped_matmul_grad_input if turned else nv.grouped_matmul
    want, lim = expected(x, spans(offsets), w, 16, turned)
    plain64.check(f(x, offsets, *w), want, lim, "y")


@pytest.mark.parametrize("first", [1, 2, 3])
@pytest.mark.parametrize("each", [5, 40, 200])
def test_scales_that_start_at_any_byte(nv, each, first):
    """One expert's share of a buffer, from any byte on; what lies before and behind does not matter."""
    g = gen(19, each, first)
    n, k = 72, 512
    q, sc, S = weights(2, n, k, 16, g)
    offsets = offsets_of([each, each + 1])
    x, dy = rand((2 * each + 1, k), g), rand((2 * each + 1, n), g)
    buffer = torch.full((sc.numel() + 8,), 0x7F, dtype=torch.uint8, device=DEV)
    moved = buffer[first:first + sc.numel()].view(sc.shape)
    moved.copy_(sc)
    assert torch.equal(nv.grouped_matmul(x, offsets, q, moved, S), nv.grouped_matmul(x, offsets, q, sc, S))
    assert torch.equal(nv.grouped_matmul_grad_input(dy, offsets, q, moved, S), nv.grouped_matmul_grad_input(dy, offsets, q, sc, S))


@pytest.mark.parametrize("each", [5, 200])
def test_last_weights_at_the_end_of_their_storage(nv, each):
    """Rows of an odd number of eights of bytes, the last of which end with a storage that goes on with other bytes."""
    g = gen(20, each)
    n, k = 33, 272
    q, sc, S = weights(2, n, k, 16, g)
    offsets = offsets_of([each, each])
    x = rand((2 * each, k), g)
    want, lim = expected(x, spans(offsets), (q, sc, S), 16, False)
    for fill in (0x00, 0xFF):
        big = torch.full((q.numel() + 64,), fill, dtype=torch.uint8, device=DEV)
        view = big[:q.numel()].view(q.shape)
        view.copy_(q)
        plain64.check(nv.grouped_matmul(x, offsets, view, sc, S), want, lim, "y")


@pytest.mark.parametrize("k", [16, 64, 80, 128, 144, 192, 256, 272, 320, 384, 448, 512, 528, 576, 784, 848])
@pytest.mark.parametrize("sizes", [[70, 64, 128, 200], [100, 1, 400, 65]])
def test_every_turn_of_the_pipeline(nv, sizes, k):
    """Contractions that end in every step of a group of four and of two, tiles of 64 and of 128 rows."""
    both(nv, sizes, 136, k, 16, torch.bfloat16, 21)


@pytest.mark.parametrize("inner", [16, 64, 144, 192, 272, 320, 448, 512])
def test_every_turn_of_the_largest_tiles(nv, inner):
    """The same for 64, 128 and 256 rows of the largest tile, by its first and last columns."""
    g = gen(22, inner)
    sizes, outer = [300, 600, 513, 130, 380, 256], 8192
    offsets = offsets_of(sizes)
    x = rand((sum(sizes), inner), g)
    for turned, f in ((False, nv.grouped_matmul), (True, nv.grouped_matmul_grad_input)):
        n, k = (inner, outer) if turned else (outer, inner)
        w = weights(len(sizes), n, k, 16, g)
        got = f(x, offsets, *w)
        for cut in (slice(0, 512), slice(outer - 512, outer)):
            part = (w[0][:, :, cut.start // 2:cut.stop // 2], w[1][:, :, cut.start // 16:cut.stop // 16], w[2]) if turned else \
                (w[0][:, cut], w[1][:, cut], w[2])
            want, lim = expected(x, spans(offsets), tuple(t.contiguous() for t in part), 16, turned)
            plain64.check(got[:, cut].contiguous(), want, lim, "y")


@pytest.mark.parametrize("k", [16, 256, 272, 512, 528, 768, 1024, 1040, 1280])
def test_every_turn_of_few_rows(nv, k):
    """Contractions of an odd and an even number of stages, shared by two fours of waves or not."""
    for n, sizes in ((48, [3, 0, 16]), (2056, [9, 12] * 16), (40, [30, 25])):
        g = gen(23, n, k)
        w = weights(len(sizes), n, k, 16, g)
        offsets = offsets_of(sizes)
        x = rand((sum(sizes), k), g)
        want, lim = expected(x, spans(offsets), w, 16, False)
        plain64.check(nv.grouped_matmul(x, offsets, *w, out_dtype=torch.float32), want, lim, "y")
