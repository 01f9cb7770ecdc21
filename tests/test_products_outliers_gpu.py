"""Activations with one value far above all others: what the others contribute stays within the sums' own bound."""
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


@pytest.mark.parametrize("block,k", [(16, 1040), (16, 1024), (32, 1024), (64, 1152)])
@pytest.mark.parametrize("m", [1, 4, 5, 40, 100, 512, 513])
def test_outlier_on_a_channel_without_weights(nv, m, block, k):
    """One channel's activations are 2^40 to 2^120 and its weights zero, so the sums are those of the others."""
    n, g = 72, workloads.generator(DEV, 531, m, block, k)
    q = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(0, 127, (n, k // block), generator=g, device=DEV, dtype=torch.uint8)
    q[:, 150] &= 15                                  # channel 301: +0
    S = torch.full((1,), 0.0371, device=DEV)
    x = torch.randn((m, k), generator=g, device=DEV)
    x[:, 301] = torch.exp2(torch.linspace(40, 120, m, device=DEV).round())
    x = x.bfloat16()
    want, bound = plain64.product(plain64.f64(x), plain64.nvfp4_values(q, sc, block))
    s = float(S.item())
    plain64.check(nv.matmul(x, q, sc, S, block=block, out_dtype=torch.float32), want * s, bound * s + 2.0 ** -23 * want.abs() * s)


@pytest.mark.parametrize("m", [8, 40, 100, 500])
def test_rows_of_every_size(nv, m):
    """Values of one row over 2^60, rows over 2^220: no bound but the sums'."""
    n, k, g = 96, 1024, workloads.generator(DEV, 532, m)
    q = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(40, 100, (n, k // 16), generator=g, device=DEV, dtype=torch.uint8)
    S = torch.ones(1, device=DEV)
    x = torch.randn((m, k), generator=g, device=DEV)
    x[:, ::3] *= 2.0 ** -30
    x[:, 1::5] *= 2.0 ** -60
    x = (x * torch.exp2(torch.linspace(-60, 100, m, device=DEV).round())[:, None]).bfloat16()
    x[m // 2] = 0
    want, bound = plain64.product(plain64.f64(x), plain64.nvfp4_values(q, sc, 16))
    # products below binary32's normal range may be lost, one quantum for each term
    plain64.check(nv.matmul(x, q, sc, S, out_dtype=torch.float32), want, bound + 2.0 ** -23 * want.abs() + k * 2.0 ** -126)


@pytest.mark.parametrize("block,k", [(16, 256), (16, 272), (32, 256), (128, 256)])
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 40, 100, 513])
def test_largest_activations(nv, m, block, k):
    """Activations of 2^126 and small scales: no sum on the way leaves binary32 where the outputs lie within it."""
    n, g = 72, workloads.generator(DEV, 533, m, block, k)
    q = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(0, 4, (n, k // block), generator=g, device=DEV, dtype=torch.uint8)
    q[:, :block // 2], sc[:, 0] = 0x77, 3            # a block of the largest values
    x = (torch.randn((m, k), generator=g, device=DEV) * 2.0 ** 123).bfloat16()
    x[:, :block] = 2.0 ** (126 if block < 128 else 122)
    S = torch.full((1,), 2.0 ** -20, device=DEV)
    want, bound = plain64.product(plain64.f64(x), plain64.nvfp4_values(q, sc, block))
    assert float(want.abs().max()) < 2.0 ** 127
    plain64.check(nv.matmul(x, q, sc, S, block=block, out_dtype=torch.float32), want * 2.0 ** -20, bound * 2.0 ** -20
                  + 2.0 ** -23 * want.abs() * 2.0 ** -20)
