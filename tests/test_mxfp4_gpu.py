"""Microscaled FP4 quantization against the nearest grid points in 64 bits, value for value."""
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


def same(nv, x):
    q, sc = nv.mx_quantize(x)
    val, codes = plain64.mx_quantize(x)
    assert torch.equal(sc.cpu(), codes)
    got = plain64.mx_values(q, sc)
    ok = (got == val) & (torch.signbit(got) == torch.signbit(val)) | (got.isnan() & val.isnan())
    assert bool(ok.all()), (~ok).nonzero()[0].tolist()
    cols = x.shape[1]
    for dt in (torch.float32, torch.bfloat16):
        back = nv.mx_dequant(q, sc, cols=cols, out_dtype=dt)
        assert back.dtype == dt and back.shape == x.shape
        b = plain64.f64(back)
        assert bool(((b == val[:, :cols]) | (b.isnan() & val[:, :cols].isnan())).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (5, 33), (7, 64), (130, 96), (64, 1000), (2, 14336),
                                       (1, 8191), (300, 40)])
def test_random(nv, rows, cols, dtype):
    g = workloads.generator(DEV, 511, rows, cols)
    x = torch.randn((rows, cols), generator=g, device=DEV) * torch.exp2(
        torch.randint(-30, 30, (rows, 1), generator=g, device=DEV).float())
    same(nv, x.to(dtype))


def test_midpoints_and_neighbours(nv):
    """Every midpoint of the grid and its neighbours, both signs, at exponents over the whole range."""
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    rows = []
    for e in range(-120, 122, 3):
        s = 2.0 ** e
        m = (mids * s).float()
        near = torch.cat([m, torch.nextafter(m, torch.tensor(float("inf"))), torch.nextafter(m, torch.zeros(()))])
        lead = torch.tensor([4.0, 7.99, 6.0, 0.0, -0.0], dtype=torch.float64) * s
        row = torch.zeros(32)
        row[:5] = lead.float()
        row[5:26] = near
        row[26:] = -near[:6]
        rows += [row, -row]
    same(nv, torch.stack(rows).to(DEV))
    same(nv, torch.stack(rows).to(torch.bfloat16).to(DEV))


def test_smallest_and_largest(nv):
    """Subnormal blocks, where the scale stops at 2^-127, zero blocks of both signs, and the largest finite values."""
    tiny = 2.0 ** -149
    x = torch.zeros((9, 32))
    x[0, :4] = torch.tensor([tiny, 3 * tiny, -tiny, 0.0])
    x[1, 3] = 2.0 ** -127
    x[2, 31] = -(2.0 ** -126)
    x[3, :] = -0.0
    x[4, :8] = torch.arange(8) * 2.0 ** -128
    x[5, 0] = torch.finfo(torch.float32).max
    x[5, 1] = -(2.0 ** 125)
    x[6, :16] = torch.arange(16) * 2.0 ** -127
    x[7, 9] = 2.0 ** -124
    x[7, 10] = 2.0 ** -126 * 0.75
    same(nv, x.to(DEV))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_blocks_without_a_maximum(nv, bad):
    g = workloads.generator(DEV, 512)
    x = torch.randn((4, 100), generator=g, device=DEV)
    x[1, 40] = bad
    x[3, 99] = bad
    same(nv, x)
    same(nv, x.to(torch.bfloat16))


@pytest.mark.parametrize("rows,cols", [(0, 64), (4, 0), (0, 0)])
def test_empty(nv, rows, cols):
    x = torch.zeros((rows, cols), device=DEV)
    q, sc = nv.mx_quantize(x)
    assert q.shape == (rows, 16 * -(-cols // 32)) and sc.shape == (rows, -(-cols // 32))
    assert nv.mx_dequant(q, sc, cols=cols).shape == (rows, cols)


def test_nothing_outside_is_written(nv):
    g = workloads.generator(DEV, 513)
    x = torch.randn((37, 70), generator=g, device=DEV)
    q0, sc0 = nv.mx_quantize(x)
    big = torch.full((37 * 48 + 64,), 171, dtype=torch.uint8, device=DEV)
    bigs = torch.full((37 * 3 + 64,), 171, dtype=torch.uint8, device=DEV)
    q, sc = big[32:32 + 37 * 48].view(37, 48), bigs[32:32 + 37 * 3].view(37, 3)
    nv.mx_quantize(x, out=(q, sc))
    assert torch.equal(q, q0) and torch.equal(sc, sc0)
    assert bool((big[:32] == 171).all()) and bool((big[32 + 37 * 48:] == 171).all())
    assert bool((bigs[:32] == 171).all()) and bool((bigs[32 + 37 * 3:] == 171).all())
