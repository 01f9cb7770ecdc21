"""8-bit integers of rows, their products and gradients, against the definitions in 64 bits."""
import numpy as np
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
    return workloads.generator(DEV, 701, *key)


def rand(shape, g, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def quantized(x):
    """(q, scales) from the definition.  (r + 0.5) s has at most 32 significant bits and x 24, so what is compared is exact."""
    x = plain64.f64(x).numpy()
    top = np.abs(x).max(-1) if x.shape[1] else np.zeros(x.shape[0])
    bad = ~np.isfinite(top)
    s = (np.where(bad, 0.0, top).astype(np.float32) * (np.float32(1) / np.float32(127))).astype(np.float64)[:, None]
    with np.errstate(invalid="ignore", divide="ignore"):
        r = np.floor(np.where(bad[:, None] | (s == 0), 0.0, x) / np.where(s == 0, 1.0, s))
        mid = (r + 0.5) * s
        r = r + np.where((x > mid) | ((x == mid) & (r % 2 == 1)), 1.0, 0.0)
    q = np.where(bad[:, None] | (s == 0), 0.0, np.clip(r, -127, 127)).astype(np.int8)
    kp = -(-x.shape[1] // 16) * 16
    out = np.zeros((x.shape[0], kp), dtype=np.int8)
    out[:, :x.shape[1]] = q
    return torch.from_numpy(out), torch.from_numpy(np.where(bad, np.nan, s[:, 0]).astype(np.float32))


def same(got, want):
    (q, s), (qw, sw) = got, want
    assert torch.equal(s.cpu().view(torch.int32).where(~s.cpu().isnan(), torch.zeros((), dtype=torch.int32)),
                       sw.view(torch.int32).where(~sw.isnan(), torch.zeros((), dtype=torch.int32)))
    assert torch.equal(s.cpu().isnan(), sw.isnan())
    off = (q.cpu() != qw).nonzero()
    assert len(off) == 0, (len(off), off[0].tolist())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 7), (5, 100), (130, 2048), (9, 2049), (4, 4096), (3, 16384), (2, 16385),
                                       (2, 50001), (7, 14330)])
def test_quantize(nv, rows, cols, dtype):
    g = gen(1, rows, cols)
    x = rand((rows, cols), g, dtype)
    same(nv.int8_quantize(x), quantized(x))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_and_their_neighbours(nv, dtype):
    """Rows whose scale is a power of two times 1, 3 or 5, with every value half way between two steps, and one ulp off."""
    rows = []
    for s in (1.0, 2.0 ** -20, 3.0 * 2.0 ** 5, 5.0, 2.0 ** 100, 2.0 ** -110, 2.0 ** -140):
        half = torch.arange(-126, 127, dtype=torch.float64).add(0.5).mul(s).to(dtype)
        up = torch.nextafter(half.float(), torch.full((), float("inf"))).to(dtype)
        down = torch.nextafter(half.float(), torch.full((), -float("inf"))).to(dtype)
        rows.append(torch.cat((half, up, down, torch.tensor([127.0 * s]).to(dtype))))
    x = torch.stack(rows).to(DEV)
    same(nv.int8_quantize(x), quantized(x))


def test_every_exponent(nv):
    """Rows from binary32's smallest numbers to its largest, and rows that span them."""
    g = gen(2)
    m = torch.rand((256, 70), generator=g, device=DEV).double() * 2 - 1
    x = (m * torch.exp2(torch.arange(-140, 116, device=DEV).double()).unsqueeze(1) * 2.0 ** 12).float()
    x[5, ::2] = 2.0 ** -149
    x[250, 3] = 3.4e38
    same(nv.int8_quantize(x), quantized(x))
    tiny = torch.zeros((4, 16), device=DEV)
    tiny[0, 3], tiny[1, 3], tiny[2, :4], tiny[3, 1] = 2.0 ** -149 * 63, 2.0 ** -149 * 64, 2.0 ** -149 * 190, -2.0 ** -149
    same(nv.int8_quantize(tiny), quantized(tiny))


@pytest.mark.parametrize("cols", [40, 5000])
def test_zeros_infinities_and_nan(nv, cols):
    x = rand((6, cols), gen(3))
    x[0] = 0.0
    x[1, 2], x[2, cols - 1], x[3, 5] = float("nan"), float("inf"), -float("inf")
    x[4] = -0.0
    same(nv.int8_quantize(x), quantized(x))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [33, 300, 2500])
def test_strided_rows(nv, cols, dtype):
    g = gen(4, cols)
    x = rand((11, cols), g, dtype)
    for first in (0, 1, 3):                              # rows that begin at any value
        big = torch.full((13, cols + 29), float("nan"), dtype=dtype, device=DEV)
        view = big[1:12, first:first + cols]
        view.copy_(x)
        same(nv.int8_quantize(view), quantized(x))
    q, s = torch.full((11, -(-cols // 16) * 16), 99, dtype=torch.int8, device=DEV), torch.empty(11, device=DEV)
    assert nv.int8_quantize(x, out=(q, s))[0] is q
    same((q, s), quantized(x))


def integers(rows, k, g, low=-127):
    q = torch.randint(low, 128, (rows, k), generator=g, device=DEV, dtype=torch.int8)
    return q, torch.rand((rows,), generator=g, device=DEV) * 0.1 + 1e-3


def product(a, b):
    """Values, and the bound of the roundings before the output's own: of the sum, of the scales' product, of theirs."""
    (aq, asc), (bq, bsc) = a, b
    y = (plain64.f64(aq) @ plain64.f64(bq).t()) * plain64.f64(asc).unsqueeze(1) * plain64.f64(bsc)
    return y, 3.01 * 2.0 ** -24 * y.abs()


ROWS = [1, 2, 3, 4, 5, 16, 17, 33, 64, 65, 128, 129, 257, 400]
SHAPES = [(m, n, k) for m in ROWS for n, k in ((77, 208), (256, 512))] + \
    [(1, 1, 16), (3, 513, 16), (300, 1, 1024), (40, 2050, 1040), (5, 300, 4112), (20, 64, 8192), (4, 300, 20000), (513, 300, 64),
     (64, 96, 14336), (33, 101, 16384), (1024, 8192, 144)]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product(nv, m, n, k, out):
    g = gen(5, m, n, k)
    a, b = integers(m, k, g), integers(n, k, g)
    plain64.check(nv.int8_matmul(a, b, out_dtype=out), *product(a, b), "y")


@pytest.mark.parametrize("m", [1, 4, 70, 300])
def test_largest_sums(nv, m):
    """The longest contraction of the largest integers stays within 32 bits."""
    k = 2 ** 17 - 16
    one = torch.ones(m, device=DEV)
    a = torch.full((m, k), -128, dtype=torch.int8, device=DEV)
    b = torch.full((40, k), -128, dtype=torch.int8, device=DEV)
    b[1] = 127
    y = nv.int8_matmul((a, one), (b, torch.ones(40, device=DEV)), out_dtype=torch.float32)
    want = torch.full((m, 40), 2.0 ** 14 * k, dtype=torch.float64)
    want[:, 1] = -128.0 * 127 * k
    assert torch.equal(y.cpu(), want.float())


@pytest.mark.parametrize("m", [2, 40, 200])
def test_a_bad_row_stays_in_its_row(nv, m):
    g = gen(6, m)
    x, w = rand((m, 100), g), nv.int8_quantize(rand((50, 100), g))
    clean = nv.int8_matmul(nv.int8_quantize(x), w)
    x[m - 1, 3] = float("inf")
    got = nv.int8_matmul(nv.int8_quantize(x), w)
    assert bool(got[m - 1].isnan().all()) and torch.equal(got[:m - 1], clean[:m - 1])


@pytest.mark.parametrize("m,n,k", [(0, 32, 64), (8, 0, 64), (8, 32, 0), (2, 5, 0)])
def test_empty(nv, m, n, k):
    a, b = nv.int8_quantize(torch.ones((m, k), device=DEV)), nv.int8_quantize(torch.ones((n, k), device=DEV))
    y = nv.int8_matmul(a, b)
    dx = nv.int8_matmul_grad_input(torch.ones((m, n), dtype=torch.bfloat16, device=DEV), *b, cols=k)
    assert y.shape == (m, n) and dx.shape == (m, k)
    if k == 0:
        assert not y.any()
    if n == 0:
        assert not dx.any()


GRADS = [(1, 1, 16), (1, 300, 64), (7, 77, 203), (64, 256, 512), (65, 130, 272), (200, 1001, 47), (300, 64, 1040), (257, 520, 500)]


def gradient(dy, q, s, cols):
    """Values and bounds: the weights are rounded to bfloat16 as operands, by at most half a step of 2^-8."""
    w = (plain64.f64(q) * plain64.f64(s).unsqueeze(1))[:, :cols]
    want, bound = plain64.product(plain64.f64(dy), w.t())
    # s q in binary32 first, then bfloat16
    return want, 1.01 * bound + (2.0 ** -8 + 2.0 ** -23) * (plain64.f64(dy).abs() @ w.abs())


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", GRADS)
def test_gradient(nv, m, n, k, out):
    g = gen(7, m, n, k)
    w = nv.int8_quantize(rand((n, k), g))
    dy = rand((m, n), g)
    got = nv.int8_matmul_grad_input(dy, *w, cols=k, out_dtype=out)
    plain64.check(got, *gradient(dy, *w, k), "dx")
    assert torch.equal(got, nv.int8_matmul_grad_input(plain64.between_nans(dy), *w, cols=k, out_dtype=out))


def test_gradient_of_powers_of_two_is_exact_but_for_its_sums(nv):
    """Scales that are powers of two leave nothing to round in the operands."""
    g = gen(8)
    q, _ = integers(96, 128, g, -128)
    s = torch.exp2(torch.randint(-8, 8, (96,), generator=g, device=DEV).float())
    dy = rand((40, 96), g)
    want, bound = plain64.product(plain64.f64(dy), (plain64.f64(q) * plain64.f64(s).unsqueeze(1)).t())
    plain64.check(nv.int8_matmul_grad_input(dy, q, s, out_dtype=torch.float32), want, bound, "dx")


def test_gradient_by_differences(nv):
    """The product is linear in A's values: one integer moved by 40 steps."""
    g = gen(9)
    m, n, k = 9, 64, 80
    (aq, asc), b = integers(m, k, g), integers(n, k, g)
    dy = rand((m, n), g)
    dx = plain64.f64(nv.int8_matmul_grad_input(dy, *b, out_dtype=torch.float32))
    bound = gradient(dy, *b, k)[1]
    y0 = plain64.f64(nv.int8_matmul((aq, asc), b, out_dtype=torch.float32))
    for i, j in ((0, 0), (4, 31), (8, 79)):
        a1 = aq.clone()
        a1[i, j] += 40 if int(aq[i, j]) < 80 else -40
        step = (plain64.f64(a1)[i, j] - plain64.f64(aq)[i, j]) * float(asc[i])
        y1 = plain64.f64(nv.int8_matmul((a1, asc), b, out_dtype=torch.float32))
        diff = ((y1 - y0) * plain64.f64(dy)).sum() / step
        noise = 4.1 * 2.0 ** -24 * ((y1.abs() + y0.abs()) * plain64.f64(dy).abs())[i].sum() / step.abs()
        assert abs(diff - dx[i, j]) <= noise + bound[i, j] + 2.0 ** -23 * dx[i, j].abs()


@pytest.mark.parametrize("m", [1, 40, 200])
def test_other_stream_captured_and_own_buffers(nv, m):
    g = gen(10, m)
    n, k = 200, 4096
    x, b = rand((m, k), g), integers(n, k, g)
    want = nv.int8_matmul(nv.int8_quantize(x), b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        later = x * 1
        for _ in range(20):
            later = later * 1
        got = nv.int8_matmul(nv.int8_quantize(later), b)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device=DEV)
    ws = torch.full((max(nv.int8_product_workspace_bytes(m, n, k), 256),), 255, dtype=torch.uint8, device=DEV)
    a = nv.int8_quantize(x)
    assert nv.int8_matmul(a, b, out=out, ws=ws) is out and torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nv.int8_matmul(nv.int8_quantize(x, out=a), b, out=out, ws=ws)
    for _ in range(3):
        x.copy_(rand((m, k), g))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, nv.int8_matmul(nv.int8_quantize(x), b))


def test_long_offsets(nv):
    """The last rows behind more than 2^32 bytes."""
    g = gen(11)
    k, m = 8192, 2 ** 19 + 100
    q = torch.zeros((m, k), dtype=torch.int8, device=DEV)
    s = torch.ones(m, device=DEV)
    q[-90:], s[-90:] = integers(90, k, g)
    b = integers(48, k, g)
    y = nv.int8_matmul((q, s), b)
    plain64.check(y[-90:], *product((q[-90:], s[-90:]), b), "y")
    assert not bool(y[:-90].any())
    y = nv.int8_matmul(b, (q, s))
    plain64.check(y[:, -90:], *product(b, (q[-90:], s[-90:])), "y")
    y = nv.int8_matmul((b[0][:2].contiguous(), b[1][:2].contiguous()), (q, s))
    plain64.check(y[:, -90:], *product((b[0][:2], b[1][:2]), (q[-90:], s[-90:])), "y")
    del q, y
    x = torch.zeros((2 ** 18 + 5, k), device=DEV)
    x[-3:] = rand((3, k), g, torch.float32)
    got = nv.int8_quantize(x)
    same((got[0][-3:], got[1][-3:]), quantized(x[-3:]))
