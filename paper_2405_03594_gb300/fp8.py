"""Linear layers in 8-bit floating point with a scale for each block of 128, on libsp (include/sp_fp8.h): the layers
that pruning leaves dense, such as the vocabulary's, and those of a small model that drafts tokens.

    m = Fp8Matrix.from_dense(w)          w [N, K] bf16, or Fp8Matrix(codes, scale) of a checkpoint
    y = m.linear(x)                      x [M, K] bf16, quantised on the way
    xq = quantize_rows(x)                once for several matrices
    y1, y2 = m1.linear(xq), m2.linear(xq)

An Fp8Matrix has a SparseMatrix's n, k and linear(), so that a Decoder takes either.  Argument marshalling only: the work
is in libsp's kernels, and PyTorch holds the buffers.  No call synchronises, so they can be captured in a CUDA graph.  Every
tensor of a call has to be on the current GPU.
"""
from __future__ import annotations

import ctypes

import torch

from . import sp
from .serve import _BF16, _F32, _on_current, _packed
from .sp import SpFp8LinearArgs, _check, _lib, _stream

BLOCK = 128  # columns of a row's block; rows and columns of a weight's
_E4M3, _U8 = torch.float8_e4m3fn, torch.uint8
_pack_linear, _linear = _packed("sp_fp8_linear", SpFp8LinearArgs)


def _blocks(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


def _rows(x: torch.Tensor, k: int | None, dev: int, name: str) -> int:
    """Checks x [rows, k] bf16 of unit column stride on GPU `dev` and returns its row stride."""
    if (x.dtype is not _BF16 or x.dim() != 2 or (k is not None and x.shape[1] != k) or x.shape[1] < 1
            or x.stride(1) != 1 or x.get_device() != dev):
        raise ValueError(f"{name}: bf16 [rows, {'columns' if k is None else k}] with unit column stride on GPU {dev} "
                         f"wanted, got {x.dtype} {list(x.shape)} on {x.device}")
    return x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1])


class Fp8Rows:
    """Quantised activations: codes (float8_e4m3fn [M, K], rows at multiples of 16 bytes) and scale (float32 [M, blocks],
    a view of one row per block)."""

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, k: int):
        self._codes, self._scale = codes, scale
        self.m, self.k = codes.shape[0], k

    @property
    def codes(self) -> torch.Tensor:
        return self._codes[:, :self.k].view(_E4M3)

    @property
    def scale(self) -> torch.Tensor:
        return self._scale[:, :self.m].t()


def quantize_rows(x: torch.Tensor, stream=None) -> Fp8Rows:
    """sp_fp8_quantize_rows: x [M, K] bf16 in e4m3, a scale for each 128 columns of a row."""
    dev = _on_current(x.get_device(), x, "x")
    stride = _rows(x, None, dev, "x")
    m, k = x.shape
    codes = torch.empty((m, (k + 15) // 16 * 16), dtype=_U8, device=x.device)
    scale = torch.empty((_blocks(k), (m + 3) // 4 * 4), dtype=_F32, device=x.device)
    _check(_lib.sp_fp8_quantize_rows(x.data_ptr(), stride, m, k, codes.data_ptr(), codes.shape[1], scale.data_ptr(),
                                     scale.shape[1], _stream(stream, dev)), "sp_fp8_quantize_rows")
    return Fp8Rows(codes, scale, k)


class Fp8Matrix:
    """A weight [N, K] in e4m3 with a scale for each 128 x 128 block: codes float8_e4m3fn (or their bytes, uint8) [N, K]
    with unit column stride, scale float32 [blocks of N, blocks of K].  Codes whose rows do not start at multiples of
    16 bytes are copied; others are used where they are."""

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor):
        if codes.dtype not in (_E4M3, _U8) or codes.dim() != 2 or min(codes.shape) < 1 or codes.stride(1) != 1 or codes.get_device() < 0:
            raise ValueError(f"codes: float8_e4m3fn [N, K] with unit column stride on a GPU wanted, got {codes.dtype} {list(codes.shape)} on {codes.device}")
        n, k = codes.shape
        if scale.dtype is not _F32 or scale.shape != (_blocks(n), _blocks(k)) or scale.get_device() != codes.get_device():
            raise ValueError(f"scale: float32 {[_blocks(n), _blocks(k)]} on {codes.device} wanted")
        codes = codes.view(_U8)
        if codes.data_ptr() % 16 or (n > 1 and codes.stride(0) % 16) or codes.stride(0) < k:
            wide = torch.zeros((n, (k + 15) // 16 * 16), dtype=_U8, device=codes.device)
            wide[:, :k] = codes
            codes = wide
        elif n == 1 and codes.stride(0) % 16:
            codes = codes.as_strided((1, k), ((k + 15) // 16 * 16, 1))
        self._codes, self._scale = codes, scale.contiguous()
        self.n, self.k, self.device = n, k, codes.get_device()
        self._ws = {}
        self._where = (codes.data_ptr(), self._scale.data_ptr())
        self._stride = codes.stride(0)

    @classmethod
    def from_dense(cls, w: torch.Tensor, stream=None) -> "Fp8Matrix":
        """sp_fp8_quantize_blocks: w [N, K] bf16."""
        dev = _on_current(w.get_device(), w, "w")
        stride = _rows(w, None, dev, "w")
        n, k = w.shape
        codes = torch.empty((n, (k + 15) // 16 * 16), dtype=_U8, device=w.device)
        scale = torch.empty((_blocks(n), _blocks(k)), dtype=_F32, device=w.device)
        _check(_lib.sp_fp8_quantize_blocks(w.data_ptr(), stride, n, k, codes.data_ptr(), codes.shape[1], scale.data_ptr(),
                                           _stream(stream, dev)), "sp_fp8_quantize_blocks")
        return cls(codes[:, :k], scale)

    @property
    def codes(self) -> torch.Tensor:
        return self._codes[:, :self.k].view(_E4M3)

    @property
    def scale(self) -> torch.Tensor:
        return self._scale

    def dense(self) -> torch.Tensor:
        """The weights that the codes stand for, float32 [N, K]."""
        s = self._scale.repeat_interleave(BLOCK, 0)[:self.n].repeat_interleave(BLOCK, 1)[:, :self.k]
        return self.codes.float() * s

    def workspace_size(self, m: int) -> int:
        b = self._ws.get(m)
        if b is None:
            c = ctypes.c_size_t()
            _check(_lib.sp_fp8_workspace_size(m, self.n, self.k, ctypes.byref(c)), "sp_fp8_workspace_size")
            b = int(c.value)
            if len(self._ws) < 256:
                self._ws[m] = b
        return b

    def linear(self, x, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """sp_fp8_linear: y = x . W^T, bf16 [M, N], of x [M, K] bf16 (rows of unit column stride) or Fp8Rows.  out: rows
        of unit column stride; workspace: workspace_size(M) bytes (uint8), zero at first as include/sp_fp8.h says."""
        dev = _on_current(self.device, self._codes, "the weight")
        if isinstance(x, Fp8Rows):
            if x.k != self.k or x._codes.get_device() != dev:
                raise ValueError(f"x: quantised [rows, {self.k}] on GPU {dev} wanted")
            m, device = x.m, x._codes.device
            rows = (0, x._codes.data_ptr(), x._scale.data_ptr())
            strides = (0, x._codes.stride(0), x._scale.stride(0))
        else:
            strides = (_rows(x, self.k, dev, "x"), 0, 0)
            m, device = x.shape[0], x.device
            rows = (x.data_ptr(), 0, 0)
        if out is None:
            out, out_stride = torch.empty((m, self.n), dtype=_BF16, device=device), self.n
        else:
            out_stride = _rows(out, self.n, dev, "out")
            if out.shape[0] != m:
                raise ValueError("x and out hold different numbers of rows")
        ws = nbytes = 0
        if workspace is None:
            nbytes = self.workspace_size(m)
            if nbytes:
                workspace = sp.workspace_for(nbytes, device, stream)
                ws, nbytes = workspace.data_ptr(), workspace.numel()
        elif workspace.dtype is not _U8 or not workspace.is_contiguous() or workspace.get_device() != dev:
            raise ValueError(f"workspace: contiguous bytes (uint8) on GPU {dev} wanted")
        else:
            ws, nbytes = workspace.data_ptr(), workspace.numel()
        _check(_linear(_pack_linear(*self._where, *rows, out.data_ptr(), self._stride, *strides, out_stride, m, self.n, self.k),
                       ws, nbytes, _stream(stream, dev)), "sp_fp8_linear")
        return out
