"""Scales in a layout that the products do not take are refused, not read as row-major ones."""
import types

import pytest
import torch


@pytest.fixture(scope="module")
def products():
    import paper_2606_07618_amd.products as products
    return products


class Device(types.SimpleNamespace):
    """What the checks look at of a contiguous device tensor."""
    is_cuda = True

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()


def tensor(*shape, dtype=torch.uint8):
    return Device(shape=torch.Size(shape), dtype=dtype)


def test_scales_by_shape(products):
    n, k = 128, 256
    x, q, S = tensor(4, k, dtype=torch.bfloat16), tensor(n, k // 2), tensor(1, dtype=torch.float32)
    assert products._nvfp4_weights(x, q, tensor(n, k // 16), S, 16) == (n, k)
    for shape in ((n * k // 16,), (n // 2, k // 8), (n, k // 16, 1)):
        with pytest.raises(ValueError):
            products._nvfp4_weights(x, q, tensor(*shape), S, 16)


@pytest.mark.gpu
def test_swizzled_scales_refused():
    import paper_2606_07618_amd as nv

    dev, n, k = torch.device("cuda:0"), 128, 256
    w, x, dy = (torch.ones((r, c), dtype=torch.bfloat16, device=dev) for r, c in ((n, k), (4, k), (4, n)))
    S = torch.full((1,), 0.5, device=dev)
    q, sc = nv.quantize_online(w, "absmax", 0.5)
    assert nv.matmul(x, q, sc, S).shape == (4, n)
    q, flat = nv.quantize_online(w, "absmax", 0.5, layout="swizzled")
    assert flat.numel() == sc.numel()
    for call in (lambda: nv.matmul(x, q, flat, S), lambda: nv.matmul_grad_input(dy, q, flat, S)):
        with pytest.raises(ValueError):
            call()
