"""Matrix products with 4-bit weights, microscaled FP4 and the gated feed-forward block: thin
wrappers of the C entry points that allocate outputs and workspaces with torch and pass raw
device pointers and the current HIP stream."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from .nvfp4 import BF16, F32, NVFP4Error, _ptr, _stream, lib

nvfp4_matmul = lib.nvfp4_matmul
nvfp4_matmul_workspace_bytes = lib.nvfp4_matmul_workspace_bytes
nvfp4_matmul_grad_input = lib.nvfp4_matmul_grad_input
nvfp4_matmul_grad_input_workspace_bytes = lib.nvfp4_matmul_grad_input_workspace_bytes
nvfp4_swiglu_ffn = lib.nvfp4_swiglu_ffn
nvfp4_swiglu_ffn_workspace_bytes = lib.nvfp4_swiglu_ffn_workspace_bytes
nvfp4_swiglu_ffn_backward = lib.nvfp4_swiglu_ffn_backward
nvfp4_swiglu_ffn_backward_workspace_bytes = lib.nvfp4_swiglu_ffn_backward_workspace_bytes
nvfp4_ffn_gradients_workspace_bytes = lib.nvfp4_ffn_gradients_workspace_bytes
mxfp4_quant = lib.mxfp4_quant
mxfp4_dequant = lib.mxfp4_dequant
mxfp4_matmul = lib.mxfp4_matmul
mxfp4_matmul_workspace_bytes = lib.mxfp4_matmul_workspace_bytes
mxfp4_matmul_grad_input = lib.mxfp4_matmul_grad_input
mxfp4_matmul_grad_input_workspace_bytes = lib.mxfp4_matmul_grad_input_workspace_bytes

MX_BLOCK = 32


def _dtype_id(dtype, what):
    if dtype == torch.bfloat16:
        return BF16
    if dtype == torch.float32:
        return F32
    raise TypeError(f"{what} must be bfloat16 or float32")


def _rows(t, what):
    """The row stride of a bfloat16 device matrix whose rows are runs of values."""
    if t.dim() != 2:
        raise ValueError(f"{what} must be 2-D")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor (the library runs on the GPU only)")
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{what} must be bfloat16")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}'s rows must be contiguous")
    if rows <= 1 or cols == 0:                      # torch gives the stride of a lone row any value
        return cols
    if t.stride(0) < cols:
        raise ValueError(f"{what}'s rows must not overlap")
    return t.stride(0)


def _same_device(t, *others):
    index = t.get_device()
    for o in others:
        if o is not None and o.get_device() != index:
            raise ValueError("all tensors must be on one device")


def _plain(t, shape, dtype, what):
    if not (t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous {dtype} device tensor {list(shape)}")


def _output(out, shape, dtype, like, what="out"):
    if out is None:
        return like.new_empty(shape, dtype=dtype)
    _plain(out, shape, dtype, what)
    _same_device(like, out)
    return out


def _workspace(nbytes, ws, like, where):
    """(pointer owner, bytes) of a workspace of at least nbytes on like's device.  The kernels write a caller's
    own from its first byte on, so it must be a run of that device's memory."""
    if nbytes < 0:
        raise NVFP4Error(int(nbytes), where)
    if nbytes == 0:
        return None, 0
    if ws is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=like.device), nbytes
    if not (ws.is_cuda and ws.is_contiguous() and ws.get_device() == like.get_device()):
        raise ValueError("ws must be a contiguous tensor on the operands' device")
    return ws, ws.numel() * ws.element_size()


def _check(rc, where):
    if rc != 0:
        raise NVFP4Error(rc, where)


# ---- microscaled FP4 -----------------------------------------------------------------------

def mx_quantize(x: torch.Tensor, out=None):
    """Microscaled FP4 (OCP MX) of a contiguous bfloat16 or float32 device matrix [rows, cols]:
    (q [rows, 16 kb] nibbles, scales [rows, kb] E8M0 codes), kb = ceil(cols / 32); the last block
    of a row is filled up with zeros.  See mxfp4_quant."""
    if x.dim() != 2:
        raise ValueError("x must be 2-D [rows, cols]")
    if not x.is_cuda:
        raise ValueError("x must be a device tensor (the library runs on the GPU only)")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    dt = _dtype_id(x.dtype, "x")
    rows, cols = x.shape
    kb = -(-cols // MX_BLOCK)
    q, sc = (None, None) if out is None else out
    q = _output(q, (rows, 16 * kb), torch.uint8, x, "q")
    sc = _output(sc, (rows, kb), torch.uint8, x, "scales")
    _check(mxfp4_quant(_ptr(x), dt, rows, cols, _ptr(q), _ptr(sc), _stream(x)), "mxfp4_quant")
    return q, sc


def _mx_pair(q, scales, what):
    if q.dim() != 2 or scales.dim() != 2:
        raise ValueError(f"{what} must be (q [rows, 16 kb], scales [rows, kb])")
    rows, kb = scales.shape
    _plain(scales, (rows, kb), torch.uint8, f"{what}'s scales")
    _plain(q, (rows, 16 * kb), torch.uint8, f"{what}'s q")
    _same_device(q, scales)
    return rows, kb


def mx_dequant(q: torch.Tensor, scales: torch.Tensor, cols: int | None = None,
               out_dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values [rows, cols] of a microscaled tensor (cols: whole blocks by default)."""
    dt = _dtype_id(out_dtype, "out_dtype")
    rows, kb = _mx_pair(q, scales, "the tensor")
    cols = MX_BLOCK * kb if cols is None else cols
    if -(-cols // MX_BLOCK) != kb:
        raise ValueError(f"cols must lie in the last of the {kb} blocks of a row")
    out = _output(out, (rows, cols), out_dtype, q)
    _check(mxfp4_dequant(_ptr(q), _ptr(scales), rows, cols, dt, _ptr(out), _stream(q)), "mxfp4_dequant")
    return out


def mx_matmul(a, b, out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
              ws: torch.Tensor | None = None) -> torch.Tensor:
    """y = A B^T [m, n] of two microscaled tensors (q, scales), A [m, k] and B [n, k]; sums in
    binary32, rounded once."""
    dt = _dtype_id(out_dtype, "out_dtype")
    (aq, asc), (bq, bsc) = a, b
    m, kb = _mx_pair(aq, asc, "a")
    n, kb2 = _mx_pair(bq, bsc, "b")
    if kb != kb2:
        raise ValueError("a and b must have rows of the same number of blocks")
    _same_device(aq, bq)
    out = _output(out, (m, n), out_dtype, aq)
    k = MX_BLOCK * kb
    ws, nbytes = _workspace(mxfp4_matmul_workspace_bytes(m, n, k), ws, aq, "mxfp4_matmul_workspace_bytes")
    _check(mxfp4_matmul(_ptr(aq), _ptr(asc), _ptr(bq), _ptr(bsc), m, n, k, dt, _ptr(out), _ptr(ws), nbytes,
                        _stream(aq)), "mxfp4_matmul")
    return out


def mx_matmul_grad_input(dy: torch.Tensor, q: torch.Tensor, scales: torch.Tensor, cols: int | None = None,
                         out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                         ws: torch.Tensor | None = None) -> torch.Tensor:
    """dx = dy B [m, cols] of a bfloat16 dy [m, n] and a microscaled B [n, cols]: the gradient of
    mx_matmul's A (straight through its quantization)."""
    dt = _dtype_id(out_dtype, "out_dtype")
    ld = _rows(dy, "dy")
    m = dy.shape[0]
    n, kb = _mx_pair(q, scales, "the weights")
    if dy.shape[1] != n:
        raise ValueError("dy must be [m, n] for weights of n rows")
    cols = MX_BLOCK * kb if cols is None else cols
    if -(-cols // MX_BLOCK) != kb:
        raise ValueError(f"cols must lie in the last of the {kb} blocks of a row")
    out = _output(out, (m, cols), out_dtype, dy)
    _same_device(dy, q)
    ws, nbytes = _workspace(mxfp4_matmul_grad_input_workspace_bytes(m, n, cols, ld), ws, dy,
                            "mxfp4_matmul_grad_input_workspace_bytes")
    _check(mxfp4_matmul_grad_input(_ptr(dy), ld, _ptr(q), _ptr(scales), m, n, cols, dt, _ptr(out), _ptr(ws), nbytes,
                                   _stream(dy)), "mxfp4_matmul_grad_input")
    return out


# ---- products with NVFP4 weights -------------------------------------------------------------

def _nvfp4_weights(x, q, scales, S, block):
    if q.dim() != 2:
        raise ValueError("q must be 2-D [n, k/2]")
    n, k = q.shape[0], q.shape[1] * 2
    _plain(q, (n, k // 2), torch.uint8, "q")
    # by shape: a flat buffer of swizzled scales may hold as many bytes
    if not (scales.is_cuda and scales.dtype == torch.uint8 and scales.is_contiguous()
            and (block <= 0 or scales.shape == (n, k // block))):
        raise ValueError("scales must be a contiguous uint8 device tensor [n, k/block], row-major")
    if not (S.is_cuda and S.dtype == torch.float32 and S.numel() >= 1):
        raise ValueError("S must be a float32 device tensor")
    _same_device(x, q, scales, S)
    return n, k


def matmul(x: torch.Tensor, q: torch.Tensor, scales: torch.Tensor, S: torch.Tensor, block: int = 16,
           out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
           ws: torch.Tensor | None = None) -> torch.Tensor:
    """y = x W^T [m, n] of a bfloat16 x [m, k] and the NVFP4 weights (q, scales, S) that quantize()
    gives for W [n, k]; weights and x enter exactly, sums in binary32, rounded once.  Recorded by autograd
    where x requires a gradient (matmul_grad_input; q, scales and S are constants), unless ``out`` is given."""
    if out is None and x.requires_grad and torch.is_grad_enabled():
        return _Matmul.apply(x, q, scales, S, block, out_dtype, ws)
    dt = _dtype_id(out_dtype, "out_dtype")
    ldx = _rows(x, "x")
    n, k = _nvfp4_weights(x, q, scales, S, block)
    m = x.shape[0]
    if x.shape[1] != k:
        raise ValueError("x must be [m, k] for weights [n, k]")
    out = _output(out, (m, n), out_dtype, x)
    ws, nbytes = _workspace(nvfp4_matmul_workspace_bytes(m, n, k), ws, x, "nvfp4_matmul_workspace_bytes")
    _check(nvfp4_matmul(_ptr(x), ldx, _ptr(q), _ptr(scales), block, _ptr(S), m, n, k, dt, _ptr(out), _ptr(ws), nbytes,
                        _stream(x)), "nvfp4_matmul")
    return out


def matmul_grad_input(dy: torch.Tensor, q: torch.Tensor, scales: torch.Tensor, S: torch.Tensor, block: int = 16,
                      out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                      ws: torch.Tensor | None = None) -> torch.Tensor:
    """dx = dy W [m, k] of a bfloat16 dy [m, n]: matmul()'s gradient with respect to x."""
    dt = _dtype_id(out_dtype, "out_dtype")
    ld = _rows(dy, "dy")
    n, k = _nvfp4_weights(dy, q, scales, S, block)
    m = dy.shape[0]
    if dy.shape[1] != n:
        raise ValueError("dy must be [m, n] for weights [n, k]")
    out = _output(out, (m, k), out_dtype, dy)
    ws, nbytes = _workspace(nvfp4_matmul_grad_input_workspace_bytes(m, n, k, ld), ws, dy,
                            "nvfp4_matmul_grad_input_workspace_bytes")
    _check(nvfp4_matmul_grad_input(_ptr(dy), ld, _ptr(q), _ptr(scales), block, _ptr(S), m, n, k, dt, _ptr(out),
                                   _ptr(ws), nbytes, _stream(dy)), "nvfp4_matmul_grad_input")
    return out


def _incoming(d):
    """A gradient as the entry points take it; autograd hands over any type, layout and alignment."""
    d = d.to(torch.bfloat16).contiguous()
    return d if d.data_ptr() % 16 == 0 else d.clone()


class _Matmul(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, q, scales, S, block, out_dtype, ws):
        ctx.save_for_backward(q, scales, S)
        ctx.block = block
        return matmul(x, q, scales, S, block, out_dtype, ws=ws)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return (matmul_grad_input(_incoming(dy), *ctx.saved_tensors, ctx.block),) + (None,) * 6


# ---- the gated feed-forward block --------------------------------------------------------------

def _ffn_operands(x, w_gate, w_up):
    ldx, ldg, ldu = _rows(x, "x"), _rows(w_gate, "w_gate"), _rows(w_up, "w_up")
    if w_gate.shape != w_up.shape or x.shape[1] != w_gate.shape[1]:
        raise ValueError("x must be [m, k], w_gate and w_up [n, k]")
    if ldg != ldu:
        raise ValueError("w_gate and w_up must have the same row stride")
    _same_device(x, w_gate, w_up)
    return x.shape[0], w_gate.shape[0], x.shape[1], ldx, ldg


def swiglu_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, save: bool = False, out=None,
               ws: torch.Tensor | None = None):
    """h = silu(x Wg^T) (x Wu^T) [m, n] in bfloat16, x [m, k], w_gate and w_up [n, k] (rows may be
    strided, the weights alike).  With ``save`` returns (h, gate, up), the pre-activations that
    swiglu_ffn_backward takes.  ``out`` may pass preallocated outputs in the same form.  Recorded by
    autograd where an operand requires a gradient, unless ``save`` (the caller's own backward) or
    ``out`` is given."""
    if out is None and not save and torch.is_grad_enabled() and (
            x.requires_grad or w_gate.requires_grad or w_up.requires_grad):
        return _SwigluFfn.apply(x, w_gate, w_up, ws)
    m, n, k, ldx, ldw = _ffn_operands(x, w_gate, w_up)
    h, gate, up = (out if save else (out, None, None)) if out is not None else (None, None, None)
    h = _output(h, (m, n), torch.bfloat16, x, "h")
    if save:
        gate = _output(gate, (m, n), torch.bfloat16, x, "gate")
        up = _output(up, (m, n), torch.bfloat16, x, "up")
    ws, nbytes = _workspace(nvfp4_swiglu_ffn_workspace_bytes(m, n, k, ldx, ldw), ws, x,
                            "nvfp4_swiglu_ffn_workspace_bytes")
    _check(nvfp4_swiglu_ffn(_ptr(x), ldx, _ptr(w_gate), _ptr(w_up), ldw, m, n, k, _ptr(h), _ptr(gate), _ptr(up),
                            _ptr(ws), nbytes, _stream(x)), "nvfp4_swiglu_ffn")
    return (h, gate, up) if save else h


def swiglu_ffn_backward(dh: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                        gate: torch.Tensor, up: torch.Tensor, need_x: bool = True, need_w: bool = True, out=None,
                        ws: torch.Tensor | None = None):
    """Gradients (dx [m, k], dw_gate, dw_up [n, k]) of swiglu_ffn in bfloat16, from dh [m, n] and the
    pre-activations it saved.  need_x / need_w: a gradient that is not needed is None and not
    computed.  ``out`` may pass preallocated gradients in the same form.  The pre-activations' gradients
    are rounded to bfloat16 once, as operands of the products."""
    m, n, k, ldx, ldw = _ffn_operands(x, w_gate, w_up)
    for t, what in ((dh, "dh"), (gate, "gate"), (up, "up")):
        _plain(t, (m, n), torch.bfloat16, what)
    if not (need_x or need_w):
        return None, None, None
    dx, dwg, dwu = out if out is not None else (None, None, None)
    dx = _output(dx, (m, k), torch.bfloat16, x, "dx") if need_x else None
    dwg = _output(dwg, (n, k), torch.bfloat16, x, "dw_gate") if need_w else None
    dwu = _output(dwu, (n, k), torch.bfloat16, x, "dw_up") if need_w else None
    _same_device(x, dh, gate, up)
    ws, nbytes = _workspace(nvfp4_ffn_gradients_workspace_bytes(m, n, k, ldx, ldw, bool(need_x), bool(need_w)), ws, x,
                            "nvfp4_ffn_gradients_workspace_bytes")
    _check(nvfp4_swiglu_ffn_backward(_ptr(dh), _ptr(x), ldx, _ptr(w_gate), _ptr(w_up), ldw, _ptr(gate), _ptr(up), m, n,
                                     k, _ptr(dx), _ptr(dwg), _ptr(dwu), _ptr(ws), nbytes, _stream(x)),
           "nvfp4_swiglu_ffn_backward")
    return dx, dwg, dwu


class _SwigluFfn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, ws):
        h, gate, up = swiglu_ffn(x, w_gate, w_up, save=True, ws=ws)
        ctx.save_for_backward(x, w_gate, w_up, gate, up)
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        x, gate, up = ctx.needs_input_grad[:3]
        dx, dwg, dwu = swiglu_ffn_backward(_incoming(dh), *ctx.saved_tensors, need_x=x, need_w=gate or up)
        return dx, dwg if gate else None, dwu if up else None, None
