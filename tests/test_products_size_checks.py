"""Checks at sizes whose products pass 63 bits or what a launch holds, on the host: they return before any launch."""
import ctypes

import pytest
import torch

A = ctypes.c_void_p(0x100000)                       # never dereferenced
M, N = 2 ** 36, 2 ** 20

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up device addresses only where no GPU is visible")


@pytest.fixture(scope="module")
def nv():
    import paper_2606_07618_amd as nv
    return nv


@pytest.mark.parametrize("m,n,k", [(4, 8, 64), (M, N, N), (2 ** 35, 2 ** 19, 2 ** 9)])
def test_backward_without_outputs(nv, m, n, k):
    """No output at all is an error, also where m n k passes 2^63."""
    rc = nv.nvfp4_swiglu_ffn_backward(A, A, k, A, A, k, A, A, m, n, k, None, None, None, A, 1 << 40, None)
    assert rc == -1
