"""The products where their kernels change form: the largest tiles with ragged edges, contractions split over workgroups,
activations of very different size in binary16, and captured graphs."""
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
    return workloads.generator(DEV, 777, *key)


def rand(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).bfloat16()


def codes(shape, lo, hi, g):
    return torch.randint(lo, hi, shape, generator=g, device=DEV, dtype=torch.uint8)


def some(rows, g, count=40):
    """Row numbers: the last ones, and others."""
    pick = torch.randint(0, rows, (count,), generator=g, device=DEV)
    return torch.cat([pick, torch.arange(max(0, rows - 8), rows, device=DEV)])


# 65, 68 and 72 blocks of a row: no whole words, whole words, whole steps
@pytest.mark.parametrize("blocks", [65, 68, 72])
def test_mx_large(nv, blocks):
    m, n, g = 2053, 4100, gen(1, blocks)
    a = codes((m, 16 * blocks), 0, 256, g), codes((m, blocks), 110, 140, g)
    b = codes((n, 16 * blocks), 0, 256, g), codes((n, blocks), 110, 140, g)
    b[1][4099, blocks - 1] = 255                                 # a block of NaN in the last row
    a[1][3, 0] = 0                                               # the smallest scale
    y = nv.mx_matmul(a, b, out_dtype=torch.float32)
    rows = some(m, g)
    want, bound = plain64.product(plain64.mx_values(a[0][rows], a[1][rows]), plain64.mx_values(*b))
    plain64.check(y[rows], want, bound, "y")
    assert bool(y[:, 4099].isnan().all()) and not bool(y[:, :4099].isnan().any())
    assert torch.equal(nv.mx_matmul(a, b)[:, :4099], y[:, :4099].bfloat16())


def test_nvfp4_large(nv):
    m, n, k, g = 2053, 1100, 1040, gen(2)
    q, sc, S = codes((n, k // 2), 0, 256, g), codes((n, k // 16), 0, 127, g), torch.tensor([0.0371], device=DEV)
    x, dy = rand((m, k), g), rand((m, n), g)
    w, s, rows = plain64.nvfp4_values(q, sc, 16), float(S.item()), some(m, g)
    for got, left, right in ((nv.matmul(x, q, sc, S), x, w), (nv.matmul_grad_input(dy, q, sc, S), dy, w.t())):
        want, bound = plain64.product(plain64.f64(left[rows]), right)
        plain64.check(got[rows], want * s, bound * s + 2.0 ** -23 * want.abs() * s)


def test_gated_large(nv):
    m, n, k, g = 2053, 1100, 1033, gen(3)
    x, wg, wu, dh = rand((m, k), g), rand((n, k), g, k ** -0.5), rand((n, k), g, k ** -0.5), rand((m, n), g)
    h, gate, up = nv.swiglu_ffn(x, wg, wu, save=True)
    rows, outs = some(m, g), some(n, g)
    want, bound = plain64.ffn(x[rows], wg, wu)
    for got, w, b in zip((h, gate, up), want, bound):
        plain64.check(got[rows], w, b)
    dx, dwg, dwu = nv.swiglu_ffn_backward(dh, x, wg, wu, gate, up)
    want, bound = plain64.ffn_grads(dh[rows], x[rows], wg, wu, gate[rows], up[rows])
    plain64.check(dx[rows], want[0], bound[0], "dx")
    want, bound = plain64.ffn_grads(dh[:, outs], x, wg[outs], wu[outs], gate[:, outs], up[:, outs])
    plain64.check(dwg[outs], want[1], bound[1], "dw_gate")
    plain64.check(dwu[outs], want[2], bound[2], "dw_up")


@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("m,n,k", [(5, 77, 4096), (17, 130, 4103), (64, 256, 8192), (130, 33, 6000)])
def test_gated_split(nv, m, n, k, save):
    g = gen(4, m, n, k)
    x, wg, wu = rand((m, k), g), rand((n, k), g, k ** -0.5), rand((n, k), g, k ** -0.5)
    got = nv.swiglu_ffn(x, wg, wu, save=save)
    want, bound = plain64.ffn(x, wg, wu)
    for a, w, b in zip(got if save else (got,), want, bound):
        plain64.check(a, w, b)


@pytest.mark.parametrize("m", [8, 40, 500])
def test_rows_of_every_size(nv, m):
    """5 to 512 rows enter in binary16, each scaled by a power of two that brings its largest value to 2^14 or more:
    what its smallest numbers, 2^-24 apart, lose of a value is at most 2^-25, 2^-39 of that largest one."""
    n, k, g = 96, 1024, gen(5, m)
    q, sc, S = codes((n, k // 2), 0, 256, g), codes((n, k // 16), 40, 100, g), torch.ones(1, device=DEV)
    x = torch.randn((m, k), generator=g, device=DEV)
    x[:, ::3] *= 2.0 ** -20
    x[:, 1::5] *= 2.0 ** -37
    x = (x * torch.exp2(torch.linspace(-120, 100, m, device=DEV).round())[:, None]).bfloat16()
    x[m // 2] = 0
    w, left = plain64.nvfp4_values(q, sc, 16), plain64.f64(x)
    want, bound = plain64.product(left, w)
    lost = 2.0 ** -39 * left.abs().amax(1)[:, None] * w.abs().sum(1)[None]
    plain64.check(nv.matmul(x, q, sc, S, out_dtype=torch.float32), want, bound + lost + 2.0 ** -23 * want.abs())


def test_many_tokens(nv):
    """Past 2^21 tokens the weights' gradients are refused and the input's is not."""
    m, n, k, g = 2 ** 21 + 8, 8, 16, gen(6)
    x0, wg, wu, dh0 = rand((8, k), g), rand((n, k), g), rand((n, k), g), rand((8, n), g)
    x, dh = torch.zeros((m, k), dtype=torch.bfloat16, device=DEV), torch.zeros((m, n), dtype=torch.bfloat16, device=DEV)
    x[-8:], dh[-8:] = x0, dh0
    h, gate, up = nv.swiglu_ffn(x, wg, wu, save=True)
    with pytest.raises(nv.NVFP4Error):
        nv.swiglu_ffn_backward(dh, x, wg, wu, gate, up)
    dx = nv.swiglu_ffn_backward(dh, x, wg, wu, gate, up, need_w=False)[0]
    want, bound = plain64.ffn_grads(dh0, x0, wg, wu, gate[-8:], up[-8:])
    plain64.check(dx[-8:], want[0], bound[0], "dx")
    assert not bool(dx[:-8].any())


@pytest.mark.parametrize("m", [1, 40, 600])
def test_captured(nv, m):
    """Replays of a captured graph on changing inputs, with eager work between, give the eager results bit for bit."""
    n, k, g = 192, 1040, gen(7, m)
    x, dy = rand((m, k), g), rand((m, n), g)
    wg, wu = rand((n, k), g, k ** -0.5), rand((n, k), g, k ** -0.5)
    q, sc, S = nv.quantize(wg, "scalesweep_mse")
    b = nv.mx_quantize(wu)

    def work():
        y = nv.matmul(x, q, sc, S)
        h, gate, up = nv.swiglu_ffn(x, wg, wu, save=True)
        return (y, h, nv.matmul_grad_input(dy, q, sc, S), nv.mx_matmul(nv.mx_quantize(x), b), nv.mx_matmul_grad_input(dy, *b),
                *nv.swiglu_ffn_backward(dy, x, wg, wu, gate, up))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = work()
    for _ in range(3):
        x.copy_(rand((m, k), g))
        dy.copy_(rand((m, n), g))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for a, w in zip(got, work()):
            assert torch.equal(a, w)
        torch.cuda.synchronize()
