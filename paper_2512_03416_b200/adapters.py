"""Projections with a low-rank adapter per request (ts_adapter_project). PyTorch supplies device memory and the stream; all
computation happens inside libtokenscale.so.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import torch

from . import binding as B
from .decoder import _check, _raw_stream

ROWS = {"plain": B.TS_ROWS_PLAIN, "qkv": B.TS_ROWS_QKV, "gate_up": B.TS_ROWS_GATE_UP}
_BF16 = (torch.bfloat16, torch.int16, torch.uint16)


def _matrix(t: torch.Tensor, shape: tuple, device, what: str) -> int:
    """Address of a contiguous bf16 tensor (or one of its bit patterns) of this shape on this device."""
    if t.shape != shape or t.dtype not in _BF16:
        raise ValueError(f"{what} must be a bf16 (or int16, uint16) tensor {list(shape)}, not {t.dtype} {list(t.shape)}")
    if t.device != device or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous and on {device}")
    return t.data_ptr()


class Adapters:
    """The adapters of one projection [N, K]: a [adapters, rank, K], b [adapters, N, rank] bf16, scale float32 [adapters] (None: 1). a and
    scale are kept, not copied; b, which has to be finite, is laid out anew here, so that an adapter whose b changes needs new Adapters. rows: which
    projection of a layer (see ts_adapter_pack): "qkv", "gate_up" (b's rows in its packed order), or "plain" for others and for adapted_project.
    status: int32, TS_DEV_TIMEOUT where a bounded wait of a projection ran out."""

    def __init__(self, a: torch.Tensor, b: torch.Tensor, scale: Optional[torch.Tensor] = None, rows: str = "plain"):
        if rows not in ROWS:
            raise ValueError(f"rows must be one of {sorted(ROWS)}")
        if not a.is_cuda or a.dim() != 3 or b.dim() != 3:
            raise ValueError("a and b must be CUDA tensors [adapters, rank, K] and [adapters, N, rank]")
        n, rank, self.k = a.shape
        self.n = b.shape[1]
        if n < 1 or rank % 8 or not 8 <= rank <= 256:
            raise ValueError("a rank is a multiple of 8 from 8 to 256")
        if scale is not None and (scale.dtype != torch.float32 or scale.device != a.device or scale.numel() != n or not scale.is_contiguous()):
            raise ValueError(f"scale must be a contiguous float32 tensor of {n} values on {a.device}")
        self.device, self.rank, self.count = a.device, rank, n
        self.rows, pa, pb = rows, _matrix(a, (n, rank, self.k), a.device, "a"), _matrix(b, (n, self.n, rank), a.device, "b")
        self.tensors = [a, scale]
        with torch.cuda.device(a.device):
            packed = [self._pack(pb, order) for order in ([B.TS_ROWS_PLAIN] if rows == "plain" else [B.TS_ROWS_PLAIN, ROWS[rows]])]
        self.args = B.ts_adapters(n, rank, pa, packed[0], packed[-1], None if scale is None else scale.data_ptr())
        self.status = torch.zeros(1, dtype=torch.int32, device=a.device)
        # behind the packing: these numbers' way to the host waits for it, and the adapters can be used on any stream
        if b.numel() and not all(math.isfinite(v) for v in torch.aminmax(b.view(torch.bfloat16))):
            raise ValueError("b must be finite: tokens of other adapters take zeros times it")

    def _pack(self, b: int, order: int) -> int:
        nbytes = B.ts_adapter_packed_bytes(self.count, self.n, self.rank)
        if nbytes == 0:
            raise ValueError("too many adapters")
        out = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        _check(B.ts_adapter_pack(b, self.count, self.n, self.rank, order, out.data_ptr(), _raw_stream(self.device.index)), "ts_adapter_pack")
        self.tensors.append(out)
        return out.data_ptr()


def stack_adapters(parts) -> tuple:
    """(a, b) of a fused projection from the (a, b) of its parts [(adapters, rank, K), (adapters, rows of the part, rank)]: a below each
    other, b on the diagonal."""
    a = torch.cat([p[0] for p in parts], 1)
    b = torch.zeros(a.shape[0], sum(p[1].shape[1] for p in parts), a.shape[1], dtype=a.dtype, device=a.device)
    row = col = 0
    for _, part in parts:
        b[:, row:row + part.shape[1], col:col + part.shape[2]] = part
        row, col = row + part.shape[1], col + part.shape[2]
    return a, b


def adapted_project(x: torch.Tensor, w: torch.Tensor, adapters: Adapters, row_tokens: Sequence[int], row_adapter: Sequence[int],
                    residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, tile_m: int = 0) -> torch.Tensor:
    """x w^T + the adapters' part (+ residual): bf16 [tokens, N]. x [tokens, K], w [N, K]; request r has the next row_tokens[r] rows of x and
    uses adapter row_adapter[r] (-1: none). tile_m: see ts_gemm_bf16."""
    dev = adapters.device
    m, k, n = x.shape[0] if x.dim() == 2 else -1, adapters.k, adapters.n
    px, pw = _matrix(x, (m, k), dev, "x"), _matrix(w, (n, k), dev, "w")
    rows = len(row_tokens)
    if len(row_adapter) != rows:
        raise ValueError("row_tokens and row_adapter must be of one length")
    pr = 0 if residual is None else _matrix(residual, (m, n), dev, "residual")
    if out is None:
        out = x.new_empty((m, n))
        po = out.data_ptr()
    else:
        po = _matrix(out, (m, n), dev, "out")
    if m == 0 and rows == 0:
        return out
    nbytes = B.ts_adapter_workspace_bytes(m, rows, adapters.count, adapters.rank)
    ws = x.new_empty((nbytes + 1) // 2)          # torch's allocator keeps it until the stream has passed this call
    _check(B.ts_adapter_project(dev.index, m, n, k, px, pw, pr, po, adapters.args, rows, row_tokens, row_adapter, ws.data_ptr(), nbytes,
                                tile_m, adapters.status.data_ptr(), _raw_stream(dev.index)), "ts_adapter_project")
    return out
