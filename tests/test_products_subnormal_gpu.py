"""Operands below bfloat16's normal range enter the products as exactly as all others."""
import pytest
import torch

import plain64

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


def tiny(m, k, g):
    """Every bfloat16 number below 2^-126, both signs: multiples of 2^-133 up to 127."""
    return (torch.randint(-127, 128, (m, k), generator=g, device=DEV).double() * 2.0 ** -133).float().to(torch.bfloat16)


def large_weights(n, k, block, g):
    """|q s| of 1024 and more, so that no product with a number of tiny() leaves the normal range."""
    q = torch.randint(0, 2, (2, n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    s = torch.randint(0, 2, (2, n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    return (q[0] + 6 + 8 * s[0]) | (q[1] + 6 + 8 * s[1]) << 4, torch.randint(0x78, 0x7F, (n, k // block), generator=g, device=DEV, dtype=torch.uint8)


@pytest.mark.parametrize("m", [1, 4, 5, 40, 100, 513])
def test_activations(nv, m):
    g = torch.Generator(DEV).manual_seed(m)
    n, k = 72, 256
    q, sc = large_weights(n, k, 16, g)
    S = torch.full((1,), 2.0 ** 90, device=DEV)
    x, dy = tiny(m, k, g), tiny(m, n, g)
    assert float(x.abs().max()) > 0
    w = plain64.nvfp4_values(q, sc, 16)
    for got, left, right in ((nv.matmul(x, q, sc, S, out_dtype=torch.float32), x, w),
                             (nv.matmul_grad_input(dy, q, sc, S, out_dtype=torch.float32), dy, w.t())):
        want, bound = plain64.product(plain64.f64(left), right)
        plain64.check(got, want * 2.0 ** 90, bound * 2.0 ** 90 + 2.0 ** -23 * want.abs() * 2.0 ** 90)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_smallest_microscaled_weights(nv, m):
    """Scales of 2^-127 and 2^-126, whose values bfloat16 holds below its normal range."""
    g = torch.Generator(DEV).manual_seed(m)
    n, k = 90, 200
    q = torch.randint(0, 256, (n, 112), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(0, 2, (n, 7), generator=g, device=DEV, dtype=torch.uint8)
    dy = (torch.randn((m, n), generator=g, device=DEV) * 2.0 ** 100).bfloat16()
    want, bound = plain64.product(plain64.f64(dy), plain64.mx_values(q, sc)[:, :k].t())
    plain64.check(nv.mx_matmul_grad_input(dy, q, sc, cols=k, out_dtype=torch.float32), want, bound)


@pytest.mark.parametrize("m", [1, 4, 5, 200])
def test_gated_block(nv, m):
    g = torch.Generator(DEV).manual_seed(m)
    n, k = 40, 128
    x = tiny(m, k, g)
    wg, wu = ((torch.randn((n, k), generator=g, device=DEV) * 2.0 ** 100).bfloat16() for _ in range(2))
    _, gate, up = nv.swiglu_ffn(x, wg, wu, save=True)
    for got, w in ((gate, wg), (up, wu)):
        plain64.check(got, *plain64.product(plain64.f64(x), plain64.f64(w)))
