"""Products with NVFP4 and microscaled FP4 weights against 64-bit products of the values they hold."""
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
    return workloads.generator(DEV, 501, *key)


def rand(shape, g, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def nvfp4_weights(n, k, block, g):
    """Random nibbles and scale codes of every exponent (0: subnormal), and a global scale."""
    q = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(0, 127, (n, k // block), generator=g, device=DEV, dtype=torch.uint8)
    return q, sc, torch.tensor([0.0371], device=DEV)


def mx_weights(n, k, g):
    kb = -(-k // 32)
    q = torch.randint(0, 256, (n, 16 * kb), generator=g, device=DEV, dtype=torch.uint8)
    if k % 32:
        tail = q.view(n, kb, 16)[:, -1]
        tail[:, -(-(k % 32) // 2):] = 0
        if k % 2:
            tail[:, k % 32 // 2] &= 15
    return q, torch.randint(110, 140, (n, kb), generator=g, device=DEV, dtype=torch.uint8)


# rows on both sides of every tile height, outputs and contractions that no tile divides
ROWS = [1, 2, 7, 16, 17, 33, 64, 65, 128, 129, 257, 400]
SHAPES = [(m, n, k) for m in ROWS for n, k in ((77, 208), (256, 512))] + \
    [(1, 1, 16), (3, 513, 16), (300, 1, 1024), (40, 2050, 1040), (5, 300, 4112), (20, 64, 8192), (513, 300, 64)]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_nvfp4_product(nv, m, n, k, out):
    g = gen(1, m, n, k)
    q, sc, S = nvfp4_weights(n, k, 16, g)
    x = rand((m, k), g)
    want, bound = plain64.product(plain64.f64(x), plain64.nvfp4_values(q, sc, 16))
    s = float(S.item())
    got = nv.matmul(x, q, sc, S, out_dtype=out)
    plain64.check(got, want * s, bound * s + 2.0 ** -23 * want.abs() * s, "y")


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(1, 130, 640), (16, 96, 1152), (50, 96, 384), (200, 130, 256)])
def test_nvfp4_blocks(nv, m, n, k, block):
    g = gen(2, m, block)
    q, sc, S = nvfp4_weights(n, k, block, g)
    x, dy = rand((m, k), g), rand((m, n), g)
    w, s = plain64.nvfp4_values(q, sc, block), float(S.item())
    want, bound = plain64.product(plain64.f64(x), w)
    plain64.check(nv.matmul(x, q, sc, S, block=block), want * s, bound * s + 2.0 ** -23 * want.abs() * s, "y")
    want, bound = plain64.product(plain64.f64(dy), w.t())
    plain64.check(nv.matmul_grad_input(dy, q, sc, S, block=block), want * s, bound * s + 2.0 ** -23 * want.abs() * s, "dx")


GRADS = [(1, 1, 16), (1, 300, 64), (7, 77, 208), (64, 256, 512), (65, 130, 272), (200, 1001, 48), (300, 64, 1040),
         (257, 520, 512)]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", GRADS)
def test_nvfp4_gradient(nv, m, n, k, out):
    g = gen(3, m, n, k)
    q, sc, S = nvfp4_weights(n, k, 16, g)
    dy = rand((m, n), g)
    s = float(S.item())
    want, bound = plain64.product(plain64.f64(dy), plain64.nvfp4_values(q, sc, 16).t())
    plain64.check(nv.matmul_grad_input(dy, q, sc, S, out_dtype=out), want * s,
                  bound * s + 2.0 ** -23 * want.abs() * s, "dx")


def test_gradient_by_differences(nv):
    """<dy, f(x + d) - f(x)> / |d| against <dx, d>: f is linear, so the difference is exact but for sums."""
    g = gen(4)
    m, n, k = 33, 96, 128
    q, sc, S = nvfp4_weights(n, k, 16, g)
    x, dy = rand((m, k), g), rand((m, n), g)
    dx = plain64.f64(nv.matmul_grad_input(dy, q, sc, S, out_dtype=torch.float32))
    y0 = plain64.f64(nv.matmul(x, q, sc, S, out_dtype=torch.float32))
    for i, j in ((0, 0), (7, 31), (32, 127)):
        x1 = x.clone()
        x1[i, j] = x[i, j] + 4.0
        step = plain64.f64(x1)[i, j] - plain64.f64(x)[i, j]
        y1 = plain64.f64(nv.matmul(x1, q, sc, S, out_dtype=torch.float32))
        diff = ((y1 - y0) * plain64.f64(dy)).sum() / step
        w = plain64.nvfp4_values(q, sc, 16) * float(S.item())
        noise = 2 * (k + 4) * plain64.SUM * ((plain64.f64(x1).abs() + plain64.f64(x).abs()) @ w.t().abs()
                                             * plain64.f64(dy).abs())[i].sum() / step.abs()
        noise += (n + 4) * plain64.SUM * (plain64.f64(dy).abs() @ w.abs())[i, j]
        assert abs(diff - dx[i, j]) <= noise


MX = [(m, n, k) for m in ROWS for n, k in ((77, 208), (256, 512))] + \
    [(1, 1, 1), (3, 513, 31), (300, 1, 1000), (40, 2050, 1056), (5, 300, 4099), (300, 260, 96), (257, 130, 2304)]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", MX)
def test_mx_product(nv, m, n, k, out):
    g = gen(5, m, n, k)
    a, b = mx_weights(m, k, g), mx_weights(n, k, g)
    want, bound = plain64.product(plain64.mx_values(*a), plain64.mx_values(*b))
    plain64.check(nv.mx_matmul(a, b, out_dtype=out), want, bound, "y")


@pytest.mark.parametrize("m,n,k", GRADS + [(65, 130, 271), (9, 40, 1)])
def test_mx_gradient(nv, m, n, k):
    g = gen(6, m, n, k)
    b = mx_weights(n, k, g)
    dy = rand((m, n), g)
    want, bound = plain64.product(plain64.f64(dy), plain64.mx_values(*b)[:, :k].t())
    for out in (torch.bfloat16, torch.float32):
        plain64.check(nv.mx_matmul_grad_input(dy, *b, cols=k, out_dtype=out), want, bound, "dx")


@pytest.mark.parametrize("m", [1, 20, 150])
def test_wide_scales(nv, m):
    """Scales over the whole E8M0 range, so long as sums stay finite; a NaN block spoils its row or column alone."""
    g = gen(7, m)
    n, k = 80, 512
    a, b = mx_weights(m, k, g), mx_weights(n, k, g)
    a[1][:, :] = torch.randint(0, 160, a[1].shape, generator=g, device=DEV, dtype=torch.uint8)
    b[1][:, :] = torch.randint(90, 200, b[1].shape, generator=g, device=DEV, dtype=torch.uint8)
    b[1][3, 5] = 255
    a[1][m - 1, 0] = 255
    want, bound = plain64.product(plain64.mx_values(*a), plain64.mx_values(*b))
    got = nv.mx_matmul(a, b, out_dtype=torch.float32)
    assert torch.equal(got.cpu().isnan(), want.isnan())
    # products below binary32's normal range may be lost, one quantum for each term
    plain64.check(got, want, bound + k * 2.0 ** -126, "y")


@pytest.mark.parametrize("m", [1, 16, 40, 150])
def test_rows_between_nans(nv, m):
    """Strided rows in a storage of NaN: nothing outside the operand enters."""
    g = gen(8, m)
    n, k = 90, 272
    q, sc, S = nvfp4_weights(n, k, 16, g)
    x = rand((m, k), g)
    xv = plain64.between_nans(x)
    assert torch.equal(nv.matmul(x, q, sc, S), nv.matmul(xv, q, sc, S))
    for width in (90, 88):
        dy = rand((m, width), g)
        dyv = plain64.between_nans(dy)
        args = (q[:width].contiguous(), sc[:width].contiguous(), S)
        assert torch.equal(nv.matmul_grad_input(dy, *args), nv.matmul_grad_input(dyv, *args))


@pytest.mark.parametrize("m", [2, 40, 150])
def test_nan_and_infinity_stay_in_their_row(nv, m):
    g = gen(9, m)
    n, k = 50, 160
    q, sc, S = nvfp4_weights(n, k, 16, g)
    x = rand((m, k), g)
    clean = nv.matmul(x, q, sc, S)
    x[m - 1, 3] = float("nan")
    x[0, 7] = float("inf")
    got = nv.matmul(x, q, sc, S)
    assert bool(got[m - 1].isnan().all()) and not bool(got[0].isfinite().any())
    assert torch.equal(got[1:m - 1], clean[1:m - 1])


@pytest.mark.parametrize("m,n,k", [(0, 32, 64), (8, 0, 64), (8, 32, 0)])
def test_empty(nv, m, n, k):
    q, sc, S = nvfp4_weights(n, k, 16, gen(10))
    x, dy = torch.ones((m, k), dtype=torch.bfloat16, device=DEV), torch.ones((m, n), dtype=torch.bfloat16, device=DEV)
    y, dx = nv.matmul(x, q, sc, S), nv.matmul_grad_input(dy, q, sc, S)
    assert y.shape == (m, n) and dx.shape == (m, k)
    a, b = mx_weights(m, k, gen(11)), mx_weights(n, k, gen(12))
    y2 = nv.mx_matmul(a, b)
    assert y2.shape == (m, n)
    if k == 0:
        assert not y.any() and not y2.any()
    if n == 0:
        assert not dx.any() and not nv.mx_matmul_grad_input(dy, *b).any()


@pytest.mark.parametrize("m", [1, 40, 200])
def test_other_stream_and_repeats(nv, m):
    """Work goes to the current stream; repeated calls give the same bits, also into one's own buffers."""
    g = gen(13, m)
    n, k = 200, 4096
    q, sc, S = nvfp4_weights(n, k, 16, g)
    a, b = mx_weights(m, k, g), mx_weights(n, k, g)
    x = rand((m, k), g)
    want, want_mx = nv.matmul(x, q, sc, S), nv.mx_matmul(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        later = x * 1
        for _ in range(20):
            later = later * 1
        got, got_mx = nv.matmul(later, q, sc, S), nv.mx_matmul(a, b)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(got_mx, want_mx)
    out = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device=DEV)
    ws = torch.full((max(nv.nvfp4_matmul_workspace_bytes(m, n, k), 256),), 255, dtype=torch.uint8, device=DEV)
    assert nv.matmul(x, q, sc, S, out=out, ws=ws) is out and torch.equal(out, want)


def test_long_offsets(nv):
    """Rows whose bytes pass 2^32: the last rows of a tall activation and of tall weights."""
    g = gen(14)
    k, m = 8192, 2 ** 18 + 300                           # 4.3 GB of bfloat16
    x = torch.zeros((m, k), dtype=torch.bfloat16, device=DEV)
    tail = rand((300, k), g)
    x[-300:] = tail
    q, sc, S = nvfp4_weights(48, k, 16, g)
    y = nv.matmul(x, q, sc, S)
    want, bound = plain64.product(plain64.f64(tail), plain64.nvfp4_values(q, sc, 16))
    f = float(S.item())
    plain64.check(y[-300:], want * f, bound * f + 2.0 ** -23 * want.abs() * f, "y")
    assert not bool(y[:-300].any())


@pytest.mark.parametrize("m", [1, 48])
def test_quantized_by_the_library(nv, m):
    """The weights and activations that the quantizers give, end to end."""
    g = gen(15, m)
    w = workloads.llm_weight(160, 512, g, DEV)
    imp = workloads.column_importance(512, g, DEV, tokens=64)
    q, sc, S = nv.quantize(w, "scalesweep_wmse", 16, weight=imp)
    x = rand((m, 512), g)
    w_hat = plain64.f64(nv.dequant(q, sc, S))
    want, bound = plain64.product(plain64.f64(x), w_hat)
    plain64.check(nv.matmul(x, q, sc, S), want, bound + 2.0 ** -22 * (plain64.f64(x).abs() @ w_hat.t().abs()), "y")
    a, b = nv.mx_quantize(x), nv.mx_quantize(w)
    want, bound = plain64.product(plain64.f64(nv.mx_dequant(*a)), plain64.f64(nv.mx_dequant(*b)))
    plain64.check(nv.mx_matmul(a, b), want, bound, "y")
