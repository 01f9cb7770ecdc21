"""The gated block's backward pass takes and asks for no workspace of a gradient that is not wanted."""
import ctypes

import pytest
import torch

A = ctypes.c_void_p(0x100000)                       # never dereferenced


@pytest.fixture(scope="module")
def nv():
    import paper_2606_07618_amd as nv
    return nv


def sizes(nv, m, n, k):
    return [nv.nvfp4_ffn_gradients_workspace_bytes(m, n, k, k, k, x, w) for x, w in ((1, 1), (1, 0), (0, 1))]


def test_sizes(nv):
    m, n, k = 8192, 14336, 4096
    both, x, w = sizes(nv, m, n, k)
    assert both == nv.nvfp4_swiglu_ffn_backward_workspace_bytes(m, n, k, k, k)
    # dx: dg and du, the turned weights; dw: dg and du turned, x turned (no part of a split here)
    assert x == 2 * (m * 2 * n + 2 * n * k) and w == 2 * (m * 2 * n + m * k) and both == x + w
    assert nv.nvfp4_ffn_gradients_workspace_bytes(-1, n, k, k, k, 1, 0) == -2


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="made-up device addresses only where no GPU is visible")
@pytest.mark.parametrize("m,n,k", [(300, 77, 200), (8192, 14336, 4096), (2 ** 21 + 8, 8, 16)])
def test_call_takes_what_it_needs(nv, m, n, k):
    def call(bytes_, dx, dw, dh=A):
        return nv.nvfp4_swiglu_ffn_backward(dh, A, k, A, A, k, A, A, m, n, k, dx, dw, dw, A, bytes_, None)

    both, x, w = sizes(nv, m, n, k)
    assert call(x - 1, A, None) == -6
    if m <= 2 ** 21:
        assert call(w - 1, None, A) == -6 and call(both - 1, A, A) == -6
    # with enough, the call passes its checks and fails at its first launch: no device here
    assert call(x, A, None) == -8
    assert m > 2 ** 21 or call(w, None, A) == -8


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(5, 40, 64), (300, 77, 200), (600, 520, 1032)])
def test_gradients_alone(nv, m, n, k):
    """Exactly the bytes asked for, with a guard behind them, give the bits of the call for all gradients."""
    g = torch.Generator("cuda").manual_seed(m)
    x, wg, wu, dh = ((torch.randn(s, generator=g, device="cuda") * 0.3).bfloat16() for s in ((m, k), (n, k), (n, k), (m, n)))
    _, gate, up = nv.swiglu_ffn(x, wg, wu, save=True)
    want = nv.swiglu_ffn_backward(dh, x, wg, wu, gate, up)
    for need_x, need_w in ((True, False), (False, True)):
        size = nv.nvfp4_ffn_gradients_workspace_bytes(m, n, k, k, k, need_x, need_w)
        store = torch.full((size + 4096,), 171, dtype=torch.uint8, device="cuda")
        got = nv.swiglu_ffn_backward(dh, x, wg, wu, gate, up, need_x=need_x, need_w=need_w, ws=store[:size])
        for a, b, need in zip(got, want, (need_x, need_w, need_w)):
            assert torch.equal(a, b) if need else a is None
        assert bool((store[size:] == 171).all())
