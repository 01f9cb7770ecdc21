"""Products of 8-bit integers whose scales' product lies outside binary32 where the output does not, in every form: the dot
products, tiles whole and split, the join of their parts."""
import pytest
import torch

import plain64
import workloads

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
LARGEST = (2.0 - 2.0 ** -7) * 2.0 ** 127                 # bfloat16's, which binary32 holds too


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


def gen(*key):
    return workloads.generator(DEV, 705, *key)


# dot products; tiles, ragged and of whole lines; contractions long enough to be split
SHAPES = [(1, 90, 208), (4, 33, 4112), (40, 77, 208), (130, 256, 512), (33, 101, 16384), (65, 64, 9600)]


def check(got, a, b):
    (aq, asc), (bq, bsc) = a, b
    sums = plain64.f64(aq) @ plain64.f64(bq).t()
    want = sums * plain64.f64(asc).unsqueeze(1) * plain64.f64(bsc)       # 2^-298 to 2^287: within 64 bits
    inside = want.abs() <= LARGEST * (1 - 2.0 ** -8)
    outside = want.abs() >= 2.0 ** 128 * (1 + 2.0 ** -20)
    g = plain64.f64(got)
    assert bool((inside | outside).any(1).all()) and bool(inside.any()) and bool((g[outside] == torch.copysign(
        torch.full_like(g[outside], float("inf")), want[outside])).all())
    # the sum, the scales' product and theirs are rounded, each by half a step at most; below the normal numbers by half of the
    # smallest one
    plain64.check(got.cpu().where(inside, torch.zeros((), dtype=got.dtype)), want.where(inside, torch.zeros((), dtype=torch.float64)),
                  (3.01 * 2.0 ** -24 * want.abs() + 2.0 ** -150).where(inside, torch.zeros((), dtype=torch.float64)), "y")


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_scales_of_every_size(nv, m, n, k, out):
    g = gen(1, m, n, k)
    aq = torch.randint(-128, 128, (m, k), generator=g, device=DEV, dtype=torch.int8)
    bq = torch.randint(-128, 128, (n, k), generator=g, device=DEV, dtype=torch.int8)
    aq[m // 2], bq[n // 2] = 0, 0                                        # sums of 0
    def scales(rows):
        e = torch.randint(-149, 128, (rows,), generator=g, device=DEV).double()
        return ((1 + torch.rand((rows,), generator=g, device=DEV).double()) * torch.exp2(e)).clamp(max=3.4e38).float()
    asc, bsc = scales(m), scales(n)
    asc[m // 3], bsc[n // 3] = 0.0, 0.0
    check(nv.int8_matmul((aq, asc), (bq, bsc), out_dtype=out), (aq, asc), (bq, bsc))


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_of_scales_beyond_either_end(nv, m, n, k):
    """Scales of 2^-76 with sums up to 2^27, of 1e20 with sums of 0 and 2^-60, of 2^110 with 2^-110."""
    ones = torch.ones((m, k), dtype=torch.int8, device=DEV)
    big = torch.full((n, k), 127, dtype=torch.int8, device=DEV)
    for sa, sb, q in ((2.0 ** -76, 2.0 ** -76, big), (1e20, 1e20, torch.zeros_like(big)), (2.0 ** 110, 2.0 ** -110, big),
                      (2.0 ** -149, 2.0 ** 126, big)):
        y = nv.int8_matmul((ones, torch.full((m,), sa, device=DEV)), (q, torch.full((n,), sb, device=DEV)), out_dtype=torch.float32)
        want = float(q[0, 0]) * k * float(torch.tensor(sa).double()) * float(torch.tensor(sb).double())
        want = torch.full((m, n), want, dtype=torch.float64)
        plain64.check(y, want, 3.01 * 2.0 ** -24 * want.abs() + 2.0 ** -150, "y")
        assert bool((y != 0).all()) == bool(q.any())


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_scales_that_are_no_numbers_stay_in_their_row_and_column(nv, m, n, k):
    g = gen(2, m, n, k)
    aq = torch.randint(1, 128, (m, k), generator=g, device=DEV, dtype=torch.int8)
    bq = torch.randint(1, 128, (n, k), generator=g, device=DEV, dtype=torch.int8)
    asc, bsc = torch.rand((m,), generator=g, device=DEV) + 0.1, torch.rand((n,), generator=g, device=DEV) + 0.1
    clean = nv.int8_matmul((aq, asc), (bq, bsc))
    asc[0], bsc[n - 1], bsc[2] = float("nan"), float("nan"), float("inf")
    y = nv.int8_matmul((aq, asc), (bq, bsc))
    assert bool(y[0].isnan().all()) and bool(y[:, n - 1].isnan().all()) and bool((y[1:, 2] == float("inf")).all())
    keep = [c for c in range(n) if c not in (2, n - 1)]
    assert torch.equal(y[1:, keep], clean[1:, keep])


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_one_far_row_or_column(nv, m, n, k, out):
    """Waves of one workgroup whose scales are all moderate beside waves whose scales are not."""
    g = gen(3, m, n, k)
    aq = torch.randint(-128, 128, (m, k), generator=g, device=DEV, dtype=torch.int8)
    bq = torch.randint(-128, 128, (n, k), generator=g, device=DEV, dtype=torch.int8)
    for row, column, size in ((m - 1, None, 2.0 ** -100), (None, n - 3, 2.0 ** 90), (0, 0, 2.0 ** -63), (m // 2, n // 2, 2.0 ** -75)):
        asc, bsc = torch.rand((m,), generator=g, device=DEV) + 0.1, torch.rand((n,), generator=g, device=DEV) + 0.1
        if row is not None:
            asc[row] *= size
        if column is not None:
            bsc[column] *= size
        check(nv.int8_matmul((aq, asc), (bq, bsc), out_dtype=out), (aq, asc), (bq, bsc))
