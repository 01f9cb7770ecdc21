"""NVFP4 scales may start at any byte: a slice of a stack of weights need not be aligned."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


@pytest.mark.parametrize("block,k", [(16, 512), (16, 288), (16, 272), (32, 512), (64, 576), (128, 384)])
@pytest.mark.parametrize("m", [1, 3, 8, 48, 130, 600])
def test_scales_at_any_byte(nv, m, block, k):
    n = 77
    g = torch.Generator(DEV).manual_seed(m + k)
    q = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
    sc = torch.randint(0, 127, (n, k // block), generator=g, device=DEV, dtype=torch.uint8)
    x, dy = (torch.randn(s, generator=g, device=DEV).bfloat16() for s in ((m, k), (m, n)))
    S = torch.full((1,), 0.0371, device=DEV)
    want = nv.matmul(x, q, sc, S, block=block), nv.matmul_grad_input(dy, q, sc, S, block=block)
    for shift in (1, 2, 3, 4, 9):
        store = torch.full((sc.numel() + 32,), 0x7E, dtype=torch.uint8, device=DEV)
        at = store[shift:shift + sc.numel()].view(sc.shape)
        at.copy_(sc)
        assert torch.equal(nv.matmul(x, q, at, S, block=block), want[0])
        assert torch.equal(nv.matmul_grad_input(dy, q, at, S, block=block), want[1])
