"""Sizes at their limits: the workspaces asked for are positive 64-bit numbers, and a size past its limit is refused."""
import pytest


@pytest.fixture(scope="module")
def nv():
    import paper_2606_07618_amd as nv
    return nv


M, N = 2 ** 36, 2 ** 20


@pytest.mark.parametrize("name,rest", [("nvfp4_matmul", ()), ("nvfp4_matmul_grad_input", (N,)), ("mxfp4_matmul", ()),
                                       ("mxfp4_matmul_grad_input", (N,)), ("nvfp4_swiglu_ffn", (N, N)),
                                       ("nvfp4_swiglu_ffn_backward", (N, N))])
def test_limits(nv, name, rest):
    need = getattr(nv, name + "_workspace_bytes")
    for k in (N - 1, N):
        assert 0 <= need(M, N, k, *rest) < 2 ** 63
    assert need(M + 1, N, N, *rest) == need(M, N + 1, N, *rest) == need(M, N, N + 1, *rest) == -2


def test_backward_needs_both_orders(nv):
    """dg and du as they lie and turned: at least twice their bytes."""
    assert nv.nvfp4_swiglu_ffn_backward_workspace_bytes(M, N, N, N, N) >= 2 * (2 * M * N * 2)
