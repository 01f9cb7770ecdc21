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


WS = 1 << 62


def test_what_a_launch_holds(nv):
    """HIP takes fewer than 2^32 threads a launch: sizes past that are refused, not sent to a launch that fails behind
    others of the same call.  (Sizes that fit go on to the next check, a missing output.)"""
    def linear(m, n, k, out=A):
        return nv.nvfp4_matmul(A, k, A, A, 16, A, m, n, k, 1, out, A, WS, None)

    # tiles of 64 x 64 to 256 x 256 outputs, 256 or 512 threads
    assert linear(2 ** 33, 64, 16) == linear(2 ** 36, 1, 16) == linear(2 ** 36, 2 ** 20, 16) == -2
    # 2048 weights of a row, 256 threads
    assert linear(1024, 2 ** 18, 2 ** 17) == linear(1024, 2 ** 20, 2 ** 20) == -2
    assert linear(2 ** 29, 64, 16, out=None) == linear(1024, 2 ** 17, 2 ** 17, out=None) == linear(4, 2 ** 20, 2 ** 20, out=None) == -1

    def grad(m, n, k, out=A):
        a = nv.nvfp4_matmul_grad_input(A, n, A, A, 16, A, m, n, k, 1, out, A, WS, None)
        assert nv.mxfp4_matmul_grad_input(A, n, A, A, m, n, k, 1, out, A, WS, None) == a
        return a

    assert grad(2 ** 33, 16, 64) == grad(64, 2 ** 19, 2 ** 18) == grad(64, 2 ** 20, 2 ** 20) == -2
    assert grad(2 ** 29, 16, 64, out=None) == grad(64, 2 ** 18, 2 ** 17, out=None) == -1

    def mx(m, n, k, out=A):
        return nv.mxfp4_matmul(A, A, A, A, m, n, k, 1, out, A, WS, None)

    assert mx(2 ** 33, 64, 32) == mx(2 ** 36, 2 ** 20, 32) == mx(2 ** 36, 1, 2 ** 20) == -2
    assert mx(2 ** 29, 64, 32, out=None) == -1

    def ffn(m, n, k, h=A):
        return nv.nvfp4_swiglu_ffn(A, k, A, A, k, m, n, k, h, None, None, A, WS, None)

    assert ffn(2 ** 33, 64, 8) == ffn(2 ** 36, 2 ** 20, 8) == -2
    assert ffn(2 ** 28, 64, 8, h=None) == -1

    def back(m, n, k, dx=A, dw=A, dh=A):
        return nv.nvfp4_swiglu_ffn_backward(dh, A, k, A, A, k, A, A, m, n, k, dx, dw, dw, A, WS, None)

    assert back(2 ** 33, 64, 8, dw=None) == back(2 ** 36, 8, 2 ** 20, dw=None) == back(2 ** 21, 2 ** 20, 2 ** 20) == -2
    assert back(2 ** 28, 64, 8, dw=None, dh=None) == -1

    def quant(rows, cols, x=A):
        a = nv.mxfp4_quant(x, 1, rows, cols, A, A, None)
        assert nv.mxfp4_dequant(A, A, rows, cols, 0, x, None) == a
        return a

    assert quant(2 ** 30, 1) == quant(2 ** 30, 32) == quant(2 ** 35 // 64, 64) == quant(1, 2 ** 35) == quant(2 ** 36, 2 ** 20) == -2
    assert quant(2 ** 30 - 64, 32, x=None) == -1
