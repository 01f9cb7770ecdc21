"""A caller's own workspace: what is no run of the operands' device memory is refused before any launch."""
import types

import pytest
import torch


@pytest.fixture(scope="module")
def products():
    import paper_2606_07618_amd.products as products
    return products


def tensor(cuda=True, contiguous=True, index=0, count=4096):
    """The attributes that the check looks at, of a tensor on any device."""
    return types.SimpleNamespace(is_cuda=cuda, is_contiguous=lambda: contiguous, get_device=lambda: index if cuda else -1,
                                 numel=lambda: count, element_size=lambda: 1)


def test_refused(products):
    x = tensor()
    for ws in (tensor(cuda=False), tensor(contiguous=False), tensor(index=1), torch.empty(4096, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            products._workspace(1024, ws, x, "f")
    ws = tensor()
    assert products._workspace(1024, ws, x, "f") == (ws, 4096)
    with pytest.raises(products.NVFP4Error):
        products._workspace(-2, ws, x, "f")


def test_not_needed(products):
    """Nothing is passed on where a call needs no workspace."""
    assert products._workspace(0, torch.empty(8, dtype=torch.uint8), tensor(), "f") == (None, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["host", "strided"])
def test_refused_by_every_call(products, kind):
    dev, m, n, k = torch.device("cuda:0"), 600, 256, 2096       # every call of these sizes takes a workspace

    def z(*shape, dtype=torch.uint8):
        return torch.zeros(shape, dtype=dtype, device=dev)

    bf16 = torch.bfloat16
    x, h, w, S = z(m, k - 1, dtype=bf16), z(m, n, dtype=bf16), z(n, k - 1, dtype=bf16), z(1, dtype=torch.float32)
    q, sc, b = z(n, k // 2), z(n, k // 16), (z(n, 33 * 16), z(n, 33))
    ws = torch.zeros(2 ** 26, dtype=torch.uint8) if kind == "host" else z(2 ** 27)[::2]
    for call in (lambda: products.matmul(z(m, k, dtype=bf16), q, sc, S, ws=ws), lambda: products.matmul_grad_input(h, q, sc, S, ws=ws),
                 lambda: products.mx_matmul((z(m, 33 * 16), z(m, 33)), b, ws=ws),
                 lambda: products.mx_matmul_grad_input(h, *b, ws=ws), lambda: products.swiglu_ffn(x, w, w, ws=ws),
                 lambda: products.swiglu_ffn_backward(h, x, w, w, h, h, ws=ws)):
        with pytest.raises(ValueError):
            call()
