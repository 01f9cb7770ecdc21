"""Products of 8-bit integers and of grouped rows at the sizes that reach every form."""
import pytest
import torch

import int8_grouped_shapes as shapes
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
    return workloads.generator(DEV, 709, *key)


def rand(shape, g):
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


@pytest.mark.parametrize("m,n,k", shapes.INT8)
def test_int8_product(nv, m, n, k):
    """Bit for bit: the sum is exact, and what is rounded after it is rounded in a known order."""
    g = gen(1, m, n, k)

    def integers(rows):
        return (torch.randint(-128, 128, (rows, k), generator=g, device=DEV, dtype=torch.int8),
                torch.rand((rows,), generator=g, device=DEV) * 0.1 + 1e-3)

    (aq, asc), (bq, bsc) = a, b = integers(m), integers(n)
    sums = aq.cpu().double() @ bq.cpu().double().t()                     # below 2^53
    want = sums.float() * (bsc.cpu() * asc.cpu().unsqueeze(1))
    assert torch.equal(nv.int8_matmul(a, b, out_dtype=torch.float32).cpu(), want)
    assert torch.equal(nv.int8_matmul(a, b).cpu(), want.to(torch.bfloat16))


def weights(experts, n, k, block, g):
    q = torch.randint(0, 256, (experts, n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(0, 127, (experts, n, k // block), generator=g, device=DEV, dtype=torch.uint8)
    return q, sc, torch.rand((experts,), generator=g, device=DEV) + 0.01


def offsets_of(sizes):
    return torch.tensor([sum(sizes[:e]) for e in range(len(sizes) + 1)], dtype=torch.int32, device=DEV)


def compare(gots, rows, sizes, w, block, turned, what):
    start = 0
    for e, size in enumerate(sizes):
        if size:
            v, s = plain64.nvfp4_values(w[0][e], w[1][e], block), float(w[2][e])
            y, bound = plain64.product(plain64.f64(rows[start:start + size]), v.t() if turned else v)
            # the sum's product with the global scale is rounded once, before the output's own rounding
            for got in gots:
                plain64.check(got[start:start + size], y * s, bound * s + 2.0 ** -24 * (y.abs() + bound) * s, (what, e))
        start += size


@pytest.mark.parametrize("sizes,n,k,block", shapes.GROUPED)
def test_few_rows(nv, sizes, n, k, block):
    g = gen(2, sum(sizes), n, k, block)
    w = weights(len(sizes), n, k, block, g)
    x = rand((sum(sizes), k), g)
    compare([nv.grouped_matmul(x, offsets_of(sizes), *w, block=block, out_dtype=t) for t in (torch.bfloat16, torch.float32)], x, sizes,
            w, block, False, "y")


@pytest.mark.parametrize("inner,block", shapes.TALL_INNER)
def test_largest_tile(nv, inner, block):
    """Blocks of 32, 64 and 128, rows of scales that are whole words and not, in both directions."""
    g = gen(3, inner, block)
    sizes = shapes.TALL
    for outer, turned, f in ((shapes.TALL_OUTER, False, nv.grouped_matmul), (shapes.TALL_OUTER, True, nv.grouped_matmul_grad_input),
                             (shapes.TALL_OUTER + block, True, nv.grouped_matmul_grad_input)):
        n, k = (inner, outer) if turned else (outer, inner)
        w = weights(len(sizes), n, k, block, g)
        x = rand((sum(sizes), inner), g)
        got = f(x, offsets_of(sizes), *w, block=block)
        for first in (0, outer - 512):                    # whole blocks
            if turned:
                first = first // block * block
                cut = (w[0][:, :, first // 2:first // 2 + 256], w[1][:, :, first // block:(first + 512) // block], w[2])
            else:
                cut = (w[0][:, first:first + 512], w[1][:, first:first + 512], w[2])
            compare([got[:, first:first + 512]], x, sizes, tuple(t.contiguous() for t in cut), block, turned, "dx" if turned else "y")
