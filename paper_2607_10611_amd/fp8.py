"""Products of FP8 block matrices: linear layers that run on the block-scaled
FP8 master weights the optimizer keeps.

A BlockMatrix holds E4M3 or E5M2 codes with one scale per 128 codes of a row:
E8M0 scales (``quantize``: activations, gradients) or FP16 ones (master weights
of madd_encode_weights, madd_step and MAdam(master_format="e4m3")).

  y = linear(x, w)                      serving: x bf16 or fp32, w a BlockMatrix
  y, xt = linear_forward(x, w)          training: also x's column blocks, which are
                                        all that the backward pass needs of x
  dx, dw = linear_backward(dy, xt, copy)  both gradients; copy: the weights' bf16
                                        compute copy
  FP8Linear(...)                        a module of the three, for autograd

Everything runs in the HIP kernels of libmadd.so on the current stream;
workspaces are torch tensors.  Quantizing is part of the product's definition: the
gradients are those of the product of the quantized matrices, with the
quantizers taken as the identity (dy, x and the weights are quantized anew along
the axis that each product sums over).  Sums are in fp32 but for the matrix
instructions' own (include/madd.h: madd_matmul_fp8): about 1.5e-5 of the result on
normally distributed values, in float32 results too.
"""
from __future__ import annotations

import math
from functools import lru_cache

import torch

from . import binding as B
from .optim import was_replaced

_FMT = {torch.float8_e4m3fn: "e4m3", torch.float8_e5m2: "e5m2"}
_DTYPE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


class BlockMatrix:
    """rows x k FP8 codes (k a multiple of 128) with their block scales.

    codes: a contiguous float8 tensor, or bytes with ``fmt`` "e4m3" or "e5m2";
    scales: rows x k/128, E8M0 bytes or FP16 codes (float16, or their 16-bit
    integer view); flat tensors of those sizes are taken with ``shape``.  cols:
    how many columns count (the rest of the last block is zeros)."""

    def __init__(self, codes, scales, fmt: str | None = None, shape=None, cols: int | None = None):
        named = _FMT.get(codes.dtype)
        if named is None and (fmt not in _DTYPE or codes.dtype not in (torch.uint8, torch.int8)):
            raise TypeError("BlockMatrix: codes must be float8_e4m3fn or float8_e5m2, or bytes "
                            f"with fmt \"e4m3\" or \"e5m2\" (got {codes.dtype}, {fmt!r})")
        if named is not None and fmt not in (None, named):
            raise ValueError(f"BlockMatrix: {codes.dtype} codes are not {fmt}")
        fmt = named or fmt
        if shape is not None:
            codes = codes.view(shape)
        if codes.dim() != 2 or codes.shape[1] % B.FP8_BLOCK:
            raise ValueError("BlockMatrix: codes must be rows of a multiple of "
                             f"{B.FP8_BLOCK} (got {tuple(codes.shape)})")
        rows, k = codes.shape
        blocks = k // B.FP8_BLOCK
        if scales.shape not in ((rows, blocks), (rows * blocks,)):
            raise ValueError(f"BlockMatrix: {rows} x {k} codes need {rows} x {blocks} scales "
                             f"(got {tuple(scales.shape)})")
        B._scale_format("BlockMatrix: scales", scales)
        if not (codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("BlockMatrix: codes and scales must be contiguous")
        if scales.dim() != 2:
            scales = scales.view(rows, blocks)
        cols = k if cols is None else cols
        if not max(k - B.FP8_BLOCK, 0) < cols <= k and not cols == k == 0:
            raise ValueError(f"BlockMatrix: cols must end in the last block of {k} (got {cols})")
        self.codes, self.scales, self.fmt, self.cols = codes, scales, fmt, cols

    @classmethod
    def _made(cls, codes, scales, fmt: str, cols: int):
        """One of quantize's own results, which need no checks."""
        m = cls.__new__(cls)
        m.codes, m.scales, m.fmt, m.cols = codes, scales, fmt, cols
        return m

    @property
    def shape(self):
        return self.codes.shape[0], self.cols

    def dequantize(self, dtype=torch.float32):
        """The values the codes and scales stand for (torch operations)."""
        rows, k = self.codes.shape
        if self.scales.element_size() == 2:
            s = self.scales.view(torch.float16).float()
        else:
            s = self.scales.view(torch.float8_e8m0fnu).float()
        q = self.codes.view(_DTYPE[self.fmt]).float().view(rows, k // B.FP8_BLOCK, B.FP8_BLOCK)
        return (q * s.unsqueeze(-1)).view(rows, k)[:, :self.cols].to(dtype)


def _empty_blocks(rows, cols, device):
    kb = -(-cols // B.FP8_BLOCK)
    return (torch.empty(rows, kb * B.FP8_BLOCK, dtype=torch.uint8, device=device),
            torch.empty(rows, kb, dtype=torch.uint8, device=device))


def _as_matrix(x):
    """x as a matrix with contiguous rows, copied only if it has none."""
    if x.dim() == 2 and x.is_contiguous():
        return x
    m = x.reshape(math.prod(x.shape[:-1]), x.shape[-1])
    if m.shape[1] > 1 and m.stride(1) != 1 or m.shape[0] > 1 and m.stride(0) < m.shape[1]:
        m = m.contiguous()
    return m


def quantize(x, fmt: str = "e4m3", rows: bool = True, cols: bool = False):
    """(blocks along x's rows, blocks along its columns) as BlockMatrix, or None
    for a direction not asked for; the second is the transposed matrix's."""
    if not (rows or cols):
        raise ValueError("quantize: nothing asked for")
    x = _as_matrix(x)
    r, c = x.shape
    q, qs = _empty_blocks(r, c, x.device) if rows else (None, None)
    t, ts = _empty_blocks(c, r, x.device) if cols else (None, None)
    B.madd_quantize_fp8(x, fmt, q, qs, t, ts)
    return (BlockMatrix._made(q, qs, fmt, c) if rows else None,
            BlockMatrix._made(t, ts, fmt, r) if cols else None)


@lru_cache(maxsize=4096)
def _workspace_bytes(which: str, m: int, n: int, k: int) -> int:
    """Bytes that a product of these sizes wants (a function of the sizes alone)."""
    return int(getattr(B.lib(), f"madd_{which}_fp8_workspace")(m, n, k))


def _workspace(which: str, m: int, n: int, k: int, device):
    nbytes = _workspace_bytes(which, m, n, k)
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes > 0 else None


def matmul(a: BlockMatrix, b: BlockMatrix, dtype=torch.bfloat16, out=None,
           accumulate: bool = False):
    """a b^T in ``dtype`` (float32 or bfloat16), or into ``out`` (added to it
    with ``accumulate``).  a's scales must be E8M0."""
    if accumulate and out is None:
        raise ValueError("matmul: accumulate needs out")
    if a.cols != b.cols:
        raise ValueError(f"matmul: operands of {a.cols} and {b.cols} columns")
    m, n, k = a.codes.shape[0], b.codes.shape[0], a.codes.shape[1]
    if out is None:
        out = torch.empty(m, n, dtype=dtype, device=a.codes.device)
    ws = _workspace("matmul", m, n, k, a.codes.device)
    B.madd_matmul_fp8(a.codes, a.fmt, a.scales, b.codes, b.fmt, b.scales, out, accumulate, ws)
    return out


def linear(x, w: BlockMatrix, dtype=torch.bfloat16, out=None):
    """x W^T: x (..., k) bf16 or fp32, k a multiple of 128, quantized to E4M3 rows
    on the way."""
    a = _as_matrix(x)
    (n, k), m, device = w.codes.shape, a.shape[0], x.device
    if a.shape[1] != w.cols:
        raise ValueError(f"linear: x and the weights have {a.shape[1]} and {w.cols} columns")
    y = torch.empty(m, n, dtype=dtype, device=device) if out is None else out
    B.madd_linear_fp8(a, w.codes, w.fmt, w.scales, y, _workspace("linear", m, n, k, device))
    return y if out is not None or x.dim() == 2 else y.view(*x.shape[:-1], n)


def linear_forward(x, w: BlockMatrix, dtype=torch.bfloat16):
    """(x W^T, x's column blocks for linear_backward): x is read once."""
    rows, cols = quantize(x, "e4m3", rows=True, cols=True)
    y = matmul(rows, w, dtype)
    return y.view(*x.shape[:-1], y.shape[1]), cols


def linear_backward(dy, xt: BlockMatrix, copy, grad_fmt: str = "e4m3", dtype=torch.bfloat16,
                    weight_dtype=torch.float32, grad_weight=None, need_dx: bool = True,
                    need_dw: bool = True):
    """(dx, dw) from dy (..., n), linear_forward's column blocks of x and the
    weights' bf16 (or fp32) compute copy (n, k).  dx is of ``dtype``; dw is of
    ``weight_dtype``, or added to ``grad_weight`` where that is given.  dy is
    quantized to grad_fmt."""
    rows, cols = quantize(dy, grad_fmt, rows=need_dx, cols=need_dw)
    dx = dw = None
    if need_dx:
        dx = matmul(rows, quantize(copy, "e4m3", rows=False, cols=True)[1], dtype)
        dx = dx.view(*dy.shape[:-1], dx.shape[1])
    if need_dw:
        dw = matmul(cols, xt, weight_dtype, out=grad_weight, accumulate=grad_weight is not None)
    return dx, dw


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, copy, codes, scales, fmt, grad_fmt):
        w = BlockMatrix(codes, scales, fmt, shape=copy.shape)
        if not copy.requires_grad:
            y, xt = linear(x, w), None
        else:
            y, xt = linear_forward(x, w)
        ctx.save_for_backward(copy, xt.codes if xt else None, xt.scales if xt else None)
        ctx.x_shape, ctx.cols, ctx.grad_fmt = x.shape, xt.cols if xt else 0, grad_fmt
        ctx.x_dtype = x.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable  # autograd does not see into the kernels
    def backward(ctx, dy):
        copy, q, s = ctx.saved_tensors
        need_dx, need_dw = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        xt = BlockMatrix(q, s, "e4m3", cols=ctx.cols) if need_dw else None
        dx, dw = linear_backward(dy, xt, copy, ctx.grad_fmt, ctx.x_dtype, copy.dtype,
                                 need_dx=need_dx, need_dw=need_dw)
        return dx.view(ctx.x_shape) if need_dx else None, dw, None, None, None, None


class FP8Linear(torch.nn.Module):
    """A bias-free linear layer whose products run on block-scaled FP8.

    ``weight`` is the bf16 compute copy (n outputs, k inputs, k a multiple of
    128) that the optimizer updates.  The forward pass runs on the FP8 master
    once ``use_master`` has been given its codes and scales (MAdam's state "q"
    and "scales" of this parameter), and on the weight quantized anew before.
    Where no gradient is wanted it is ``linear``; it has first derivatives only."""

    def __init__(self, in_features: int, out_features: int, grad_fmt: str = "e4m3", device=None):
        super().__init__()
        if in_features % B.FP8_BLOCK:
            raise ValueError(f"FP8Linear: in_features must be a multiple of {B.FP8_BLOCK} "
                             f"(got {in_features})")
        if grad_fmt not in _DTYPE:
            raise ValueError(f"FP8Linear: grad_fmt must be one of {sorted(_DTYPE)}, "
                             f"not {grad_fmt!r}")
        w = torch.randn(out_features, in_features, device=device) * in_features ** -0.5
        self.weight = torch.nn.Parameter(w.to(torch.bfloat16))
        self.grad_fmt = grad_fmt
        self._master = self._given = None

    def use_master(self, codes, scales, fmt: str = "e4m3"):
        """Run the forward pass on this block-scaled master (its storage is read
        at every call, so the optimizer's in-place updates are seen).  After
        MAdam.load_state_dict, which replaces the state's tensors, call it again:
        until then the forward pass raises.  Loading the layer's own weight from a
        state dict ends it, and the weight is read again."""
        w = BlockMatrix(codes, scales.view(torch.int16), fmt, shape=self.weight.shape)
        self._master, self._given = (w.codes, w.scales, fmt), (codes, scales)

    def _load_from_state_dict(self, state_dict, prefix, *args, **kwargs):
        super()._load_from_state_dict(state_dict, prefix, *args, **kwargs)
        if prefix + "weight" in state_dict:
            self._master = self._given = None

    def forward(self, x):
        if self._master is not None:
            if any(map(was_replaced, self._given)):
                raise RuntimeError("FP8Linear: the optimizer has replaced this master "
                                   "(load_state_dict); call use_master with the new one")
            codes, scales, fmt = self._master
        else:
            w = quantize(self.weight.detach(), "e4m3")[0]
            codes, scales, fmt = w.codes, w.scales, "e4m3"
        # (within a Function a parameter requires gradients also where none are recorded)
        if not (torch.is_grad_enabled() and (x.requires_grad or self.weight.requires_grad)):
            return linear(x, BlockMatrix._made(codes, scales, fmt, self.weight.shape[1]))
        return _Linear.apply(x, self.weight, codes, scales, fmt, self.grad_fmt)
